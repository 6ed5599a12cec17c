"""mpk_rows_logprobs on the GPU against 64-bit results."""
import math
import random

import pytest
import torch

import paper_2512_22219_amd as M
from tests.rows_util import F32_HALF, RowsModel, workspace

pytestmark = pytest.mark.gpu
_models = {}


def _graph(vocab):
    if vocab not in _models:
        _models[vocab] = RowsModel(vocab=vocab, layers=1, batch=1)
    return _models[vocab].graph


def _call(vocab, x, tokens, n_top, entropy=True, stream=None):
    R, dev = x.shape[0], x.device
    lp = torch.full((R,), 9.0, device=dev) if tokens is not None else None
    en = torch.full((R,), 9.0, device=dev) if entropy else None
    ids, tops = torch.full((R, n_top), 9, dtype=torch.int32, device=dev), torch.full((R, n_top), 9.0, device=dev)
    kind = M.ROWS_F32 if x.dtype == torch.float32 else M.ROWS_BF16
    g, work = _graph(vocab), workspace()
    ptr = lambda t: t.data_ptr() if t is not None else 0  # noqa: E731
    g.rows_logprobs(R, x.data_ptr(), kind, x.stride(0), ptr(tokens), n_top, ptr(lp), ptr(en), ptr(ids), ptr(tops), work.data_ptr(),
                    torch.cuda.current_stream().cuda_stream if stream is None else stream)
    torch.cuda.synchronize()
    return lp, en, ids, tops


def _check(vocab, x, tokens, n_top):
    lp, en, ids, tops = _call(vocab, x, tokens, n_top)
    _graph(vocab).status()
    p = torch.log_softmax(x.double(), -1)
    gap = x.double() - x.double().amax(-1, keepdim=True)
    # the sum: an exponential each (two steps) and n / 256 additions in a row, then the joins; a log and two subtractions
    total = (vocab / 256 + 64) * F32_HALF
    tol = lambda at: total + 4 * F32_HALF * at.abs().nan_to_num(0.0, 0.0, 0.0)  # noqa: E731

    def near(got, want, bound):
        fine = torch.isfinite(want)
        assert torch.equal(got[~fine], want[~fine].float())
        assert ((got.double() - want).abs() <= bound)[fine].all(), ((got.double() - want).abs() - bound)[fine].max()

    rows = torch.arange(x.shape[0], device=x.device)
    asked = tokens.long().clamp(min=0)
    want = torch.where(tokens >= 0, p[rows, asked], 0.0)
    near(lp, want, tol(gap[rows, asked]) + 4 * F32_HALF * want.abs().nan_to_num(0.0, 0.0, 0.0))
    h = -(p.exp() * p.clamp(min=-1e4)).sum(-1)
    near(en, h, total * (2 * h + 2) + 8 * F32_HALF * (1 + h))
    order = x.double().sort(dim=-1, descending=True, stable=True)
    best = order.indices[:, :n_top]
    assert torch.equal(ids.long(), best)
    near(tops, p.gather(1, best), tol(gap.gather(1, best)) + 4 * F32_HALF * p.gather(1, best).abs().nan_to_num(0.0, 0.0, 0.0))


def _inputs(rows, vocab, dtype, seed, std=3.0, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty(rows, vocab + pad, device="cuda").normal_(0, std, generator=gen)
    if pad:
        x[:, vocab:] = float("nan")   # (what lies between rows is nobody's)
    tokens = torch.randint(vocab, (rows,), generator=gen, device="cuda").to(torch.int32)
    return x.to(dtype)[:, :vocab], tokens


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,n_top,pad", [
    (1, 1, 1, 0), (3, 2, 2, 1), (2, 31, 31, 0), (5, 63, 32, 2), (4, 64, 5, 0), (7, 257, 20, 3), (2, 1024, 32, 0), (300, 1000, 4, 8),
    (1, 4097, 32, 0), (1, 30011, 20, 1), (9, 30011, 1, 5), (1, 151936, 20, 0), (3, 151936, 32, 7), (16, 128256, 5, 0), (70, 50257, 20, 0),
    (1100, 2047, 8, 1), (600, 8193, 32, 0), (2, 32000, 0, 0)])
def test_random_rows(rows, vocab, n_top, pad, dtype):
    x, tokens = _inputs(rows, vocab, dtype, rows + vocab, pad=pad)
    _check(vocab, x, tokens, n_top)


@pytest.mark.parametrize("rows", [1023, 1024, 1025, 2047, 2048])
def test_as_many_rows_as_are_cut_and_more(rows):
    """Rows of a call are cut into runs up to 1023 of them; each has a counter of its own, twice in a row."""
    x, tokens = _inputs(rows, 8193, torch.float32, rows)
    _check(8193, x, tokens, 8)
    first, second = _call(8193, x, tokens, 8), _call(8193, x, tokens, 8)
    assert all(torch.equal(a, b) for a, b in zip(first, second))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [1, 3])
def test_rows_at_any_address(offset, dtype):
    flat, _ = _inputs(1, 5 * 30020 + 8, dtype, 3)
    x = flat[0, offset:offset + 5 * 30019].view(5, 30019)[:, :30011]
    _check(30011, x, torch.tensor([0, 30010, -1, 7, 15000], dtype=torch.int32, device="cuda"), 20)


@pytest.mark.parametrize("kind", ["equal", "two", "rising", "falling", "steps", "zeros", "one lane", "far"])
@pytest.mark.parametrize("rows,vocab", [(1, 151936), (2, 30011), (40, 1000), (513, 4099)])
def test_ties_and_orders(kind, rows, vocab):
    i = torch.arange(vocab, device="cuda").expand(rows, vocab)
    x = {"equal": i * 0.0 + 1.5, "two": (i % 2) * 1.0, "rising": i * 1e-4, "falling": -i * 1e-4, "steps": -((i % 97) // 13).float(),
         "zeros": torch.where(i % 3 == 0, -0.0, 0.0), "one lane": torch.where(i % 256 == 255, 8.0, 0.0) + i * 1e-6,
         "far": torch.where(i == vocab - 1, 3e38, -3e38)}[kind].float().contiguous()
    tokens = torch.arange(rows, device="cuda").to(torch.int32) * (vocab // rows)
    if kind == "far":   # (a distance of 6e38 is -inf in 32 bits, and so is its logprob's)
        lp, en, ids, tops = _call(vocab, x, tokens, 20)
        _graph(vocab).status()
        assert (en == 0).all() and (ids[:, 0] == vocab - 1).all() and (tops[:, 0] == 0).all() and (lp[0] < -1e38)
        assert torch.equal(ids[:, 1:], torch.arange(19, device="cuda", dtype=torch.int32).expand(rows, 19))
        return
    _check(vocab, x, tokens, 20)


@pytest.mark.parametrize("seed", range(40))
def test_drawn_rows(seed):
    rng = random.Random(seed)
    vocab = rng.choice([rng.randint(1, 300), rng.randint(300, 9000), rng.randint(9000, 160000)])
    rows = rng.choice([1, 2, rng.randint(3, 60), max(1, min(rng.randint(60, 3000), (1 << 25) // vocab))])
    dtype, pad, n_top = rng.choice([torch.float32, torch.bfloat16]), rng.choice([0, 0, 1, 5, 64]), min(vocab, rng.choice([0, 1, 3, 20, 32]))
    x, tokens = _inputs(rows, vocab, dtype, seed, std=rng.choice([0.01, 3.0, 40.0]), pad=pad)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if rng.random() < 0.4:   # tokens ruled out, up to all but two in a hundred; the first token stays
        out = torch.rand(rows, vocab, generator=gen, device="cuda") < rng.choice([0.1, 0.9, 0.98])
        out[:, 0] = False
        x.masked_fill_(out, -math.inf)
    if rng.random() < 0.3:
        tokens[torch.rand(rows, generator=gen, device="cuda") < 0.5] = -1
    _check(vocab, x, tokens, n_top)


def test_rows_far_apart():
    """Row strides of 2^31 elements: the third row begins past 2^32."""
    vocab, stride = 5000, 1 << 31
    x, tokens = _inputs(3, vocab, torch.bfloat16, 4)
    far = torch.empty(2 * stride + vocab, dtype=torch.bfloat16, device="cuda").as_strided((3, vocab), (stride, 1))
    far.copy_(x)
    for a, b in zip(_call(vocab, x, tokens, 20), _call(vocab, far, tokens, 20)):
        assert torch.equal(a, b)
    _check(vocab, far, tokens, 20)


def test_a_million_rows():
    vocab, rows = 64, (1 << 20) + 3
    x, tokens = _inputs(rows, vocab, torch.bfloat16, 5)
    _check(vocab, x, tokens, 3)


@pytest.mark.parametrize("n_top", [1, 6, 20, 32])
@pytest.mark.parametrize("rows,vocab,shift", [(1, 151936, 0.0), (3, 60001, -0.5), (90, 60001, -2.0), (300, 30011, 1.0), (2050, 5000, -9.5)])
def test_many_equal_logits(rows, vocab, shift, n_top):
    """Logits in steps of a quarter, so that many are equal to the last alternative; the same bits however the call went."""
    x, tokens = _inputs(rows, vocab, torch.float32, 12, std=0.5)
    x = ((4 * x).round() / 4 + shift).to(torch.bfloat16)
    _check(vocab, x, tokens, n_top)
    first = _call(vocab, x, tokens, n_top)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, _call(vocab, x, tokens, n_top)))


@pytest.mark.parametrize("rows,vocab", [(1, 30011), (3, 8000), (2100, 1000)])
@pytest.mark.parametrize("level", [1e4, 1.0e6, 1.1e6, 3e7, 1e12, 1e30])
def test_large_logits(level, rows, vocab):
    """Around `level`, in steps of its last place: a row may rise from small logits to these."""
    x, tokens = _inputs(rows, vocab, torch.float32, 8)
    step = torch.finfo(torch.float32).eps * level
    x = (level + (x * max(1.0, 2 * step)).round())
    x[0, : vocab // 3] = torch.arange(vocab // 3, device="cuda") * 1e-3
    x[rows - 1] = -x[rows - 1]
    _check(vocab, x, tokens, 20)


@pytest.mark.parametrize("vocab", [1000, 30011, 151936])
def test_ruled_out_tokens(vocab):
    x, tokens = _inputs(6, vocab, torch.float32, 1)
    x[0, : vocab - 7] = -math.inf          # seven left, of twenty asked for
    x[1, 1:] = -math.inf                   # one left: certain
    x[2, ::2] = -math.inf
    x[3, : vocab // 2] = torch.finfo(torch.float32).min   # the type's lowest value is a logit like any other
    tokens[0], tokens[1], tokens[2] = 0, 0, 1
    _check(vocab, x, tokens, 20)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [40, 30011, 151936])
def test_rows_without_a_distribution(vocab, dtype):
    x, tokens = _inputs(5, vocab, dtype, 2)
    x = x.clone()
    x[0, vocab - 1] = math.nan
    x[1, 0] = math.inf
    x[2] = -math.inf
    x[3, 5], x[3, 6] = math.nan, math.inf
    tokens[2] = -1
    lp, en, ids, tops = _call(vocab, x, tokens, 20)
    _graph(vocab).status()
    assert lp[[0, 1, 3]].isnan().all() and lp[2] == 0 and en[:4].isnan().all() and (ids[:4] == -1).all() and tops[:4].isnan().all()
    _check(vocab, x[4:], tokens[4:], 20)


def test_tokens_out_of_range_are_reported():
    x, tokens = _inputs(4, 1000, torch.float32, 4)
    for bad in (1000, -2, 2 ** 31 - 1):
        tokens[2] = bad
        lp, en, ids, tops = _call(1000, x, tokens, 3)
        with pytest.raises(M.MpkError, match="sequence 2 has token") as e:
            _graph(1000).status()
        assert e.value.status == M.MPK_ERR_DEVICE
        _graph(1000).reset()
        assert lp[2].isnan() and torch.isfinite(lp[[0, 1, 3]]).all() and torch.isfinite(en).all()
    tokens[2] = -1
    _check(1000, x, tokens, 3)


@pytest.mark.parametrize("rows,vocab", [(4, 1000), (3, 30011), (2100, 300)])
def test_a_token_out_of_range_is_reported_with_its_row(rows, vocab):
    x, tokens = _inputs(rows, vocab, torch.float32, 4)
    tokens[rows - 1] = -2
    _call(vocab, x, tokens, 3)
    with pytest.raises(M.MpkError, match=rf"token -2 outside \[-1, vocab\).*row {rows - 1} of a call") as e:
        _graph(vocab).status()
    assert e.value.status == M.MPK_ERR_DEVICE
    _graph(vocab).reset()
    tokens[rows - 1] = -1
    _check(vocab, x, tokens, 3)


@pytest.mark.parametrize("rows,vocab", [(2, 151936), (700, 3001)])
def test_parts_of_the_answer_alone(rows, vocab):
    x, tokens = _inputs(rows, vocab, torch.bfloat16, 5)
    lp, en, ids, tops = _call(vocab, x, tokens, 7)
    a = _call(vocab, x, None, 7, entropy=False)
    b = _call(vocab, x, tokens, 0, entropy=False)
    c = _call(vocab, x, None, 0)
    assert torch.equal(a[2], ids) and torch.equal(a[3], tops) and torch.equal(b[0], lp) and torch.equal(c[1], en)
    d = _call(vocab, x, None, 0, entropy=False)
    assert d[0] is None and d[1] is None


def test_captured_and_on_another_stream():
    vocab = 30011
    x, tokens = _inputs(9, vocab, torch.float32, 6)
    g, work = _graph(vocab), workspace()
    lp, en = torch.empty(9, device="cuda"), torch.empty(9, device="cuda")
    ids, tops = torch.empty(9, 20, dtype=torch.int32, device="cuda"), torch.empty(9, 20, device="cuda")

    def call(stream):
        g.rows_logprobs(9, x.data_ptr(), M.ROWS_F32, vocab, tokens.data_ptr(), 20, lp.data_ptr(), en.data_ptr(), ids.data_ptr(),
                        tops.data_ptr(), work.data_ptr(), stream)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(torch.cuda.current_stream().cuda_stream)
    side = torch.cuda.Stream()
    for i in range(4):
        x.copy_(_inputs(9, vocab, torch.float32, 10 + i)[0])
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (lp, en, ids, tops)]
        for t in (lp, en, ids, tops):
            t.zero_()
        side.wait_stream(torch.cuda.current_stream())
        call(side.cuda_stream)
        side.synchronize()
        assert all(torch.equal(u, w) for u, w in zip(got, (lp, en, ids, tops)))
        p = torch.log_softmax(x.double(), -1)
        assert torch.equal(ids.long(), x.double().sort(dim=-1, descending=True, stable=True).indices[:, :20])
        assert (tops - p.gather(1, ids.long())).abs().max() < 1e-4
    g.status()


def test_what_a_server_decodes_is_scored_through_another_graph():
    """A serving graph refuses the calls on rows; any other graph of the vocabulary takes the logits that its server left."""
    m = RowsModel(n_q=4, n_kv=2, d=64, batch=2, layers=2, vocab=9001, max_seq=64, page=16, pages=20, fill=0.0)
    ptrs = {n: t.data_ptr() for n, t in m.outer.items()}
    ptrs["layers"] = [{n: t.data_ptr() for n, t in w.items()} for w in m.w]
    served = M.compile_graph(m.shape, ptrs, (m.k.data_ptr(), m.v.data_ptr()), fusion=31, transitive_reduction=1, kv_page_size=16, kv_pages=20,
                             serving=1, greedy_loop=1)
    server = served.serve(4, 8, 8)
    for prompt in ([5, 900, 17], [8000, 1, 2]):
        server.submit(prompt, 8)
    server.run(10)   # (three tokens of the prompt; the eighth new one of both sequences is what the last iteration sampled)
    torch.cuda.synchronize()
    server.status()
    last = server.state()["tokens"]
    lp, en, work = torch.empty(2, device="cuda"), torch.empty(2, device="cuda"), workspace()
    tops, best = torch.empty(2, 5, device="cuda"), torch.empty(2, 5, dtype=torch.int32, device="cuda")
    with pytest.raises(M.MpkError, match="server"):
        served.rows_logprobs(2, server.logits_ptr(), M.ROWS_F32, 9001, 0, 5, 0, en.data_ptr(), best.data_ptr(), tops.data_ptr(), work.data_ptr())
    tokens = m.ints(last)
    m.graph.rows_logprobs(2, server.logits_ptr(), M.ROWS_F32, 9001, tokens.data_ptr(), 5, lp.data_ptr(), en.data_ptr(), best.data_ptr(),
                          tops.data_ptr(), work.data_ptr())
    m.status()
    server.status()
    assert best[:, 0].tolist() == last   # (greedy: what was sampled is the most probable)
    assert torch.isfinite(lp).all() and torch.equal(lp, tops[:, 0]) and (en > 0).all()
    server.destroy()
