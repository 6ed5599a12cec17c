"""mpk_rows_append and mpk_rows_attend on the GPU against 64-bit results."""
import random
from types import SimpleNamespace

import pytest
import torch

import paper_2512_22219_amd as M
from tests.rows_util import BF16_HALF, F32_HALF, RowsModel, append_exact, attend_exact, workspace

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.contiguous().view(torch.int16)


def _begin(lens, first=0):
    out = [first]
    for n in lens:
        out.append(out[-1] + n)
    return out


# rows of a sequence: none, one, a few, a tile and around it; first rows and rows behind the last left alone
APPEND = [
    dict(n_q=4, n_kv=2, d=64, lens=[1], pos=[0], slots=None),
    dict(n_q=8, n_kv=8, d=128, lens=[3, 0, 1], pos=[7, 191, 191], slots=[2, 0, 1], qk_norm=True),
    dict(n_q=16, n_kv=2, d=64, lens=[33, 64, 5, 90], pos=[0, 128, 60, 101], slots=[3, 2, 1, 0], theta=1e6, first=2, behind=3),
    dict(n_q=16, n_kv=2, d=128, lens=[0, 17], pos=[5, 11], slots=None, qk_norm=True, page=8, pages=101, behind=5),
    dict(n_q=4, n_kv=1, d=128, lens=[100, 100, 92, 1], pos=[92, 0, 100, 64], slots=[1, 0, 3, 2], page=64, pages=13, first=1),
    dict(n_q=32, n_kv=8, d=128, lens=[300], pos=[3700], slots=[1], max_seq=4096, batch=2, qk_norm=True, theta=5e5),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad", [0, 24])
@pytest.mark.parametrize("case", APPEND)
def test_append(case, pad, dtype):
    c = dict(case)
    lens, pos, slots, first, behind = c.pop("lens"), c.pop("pos"), c.pop("slots"), c.pop("first", 0), c.pop("behind", 0)
    m = RowsModel(**c)
    begin = _begin(lens, first)
    rows, heads = begin[-1] + behind, m.n_q + 2 * m.n_kv
    x = m.normal(rows, heads * m.d + pad, dtype=torch.float32).to(dtype)
    q_out = m.normal(rows, m.n_q * m.d + pad)
    q0, k0, v0 = q_out.clone(), m.k.clone(), m.v.clone()
    m.append(1, begin, slots, pos, x, q_out)
    m.status()
    k1, v1, q1 = k0.clone(), v0.clone(), q0.clone()
    for i, (n, p) in enumerate(zip(lens, pos)):
        if not n:
            continue
        r = slice(begin[i], begin[i + 1])
        at = torch.arange(p, p + n, device=m.dev)
        q, k, v, q_size, k_size = append_exact(m, 1, at, x[r, : heads * m.d])
        slot = slots[i] if slots else i
        # norm (d squares, root, two products) and rotation (two products, the angle's sine) in 32 bits, one rounding
        noise = (m.d / 4 + 16) * F32_HALF
        for got, want, size in ((q_out[r, : m.n_q * m.d].view(n, m.n_q, m.d), q, q_size),
                                (m.cached(m.k, 1, slot, p + n)[:, p:].transpose(0, 1), k, k_size),
                                (m.cached(m.v, 1, slot, p + n)[:, p:].transpose(0, 1), v, torch.zeros_like(v))):
            far = (got.double() - want).abs() - (BF16_HALF * want.abs() + noise * size)
            assert far.max() <= 0, far.max()
        q1[r, : m.n_q * m.d] = q_out[r, : m.n_q * m.d]
        for cache, new in ((k1, m.k), (v1, m.v)):   # the rows written, the others as they were
            if m.page:
                pg = m.table[slot].long()[at // m.page]
                cache[1][pg, :, at % m.page] = new[1][pg, :, at % m.page]
            else:
                cache[1, slot, :, p:p + n] = new[1, slot, :, p:p + n]
    assert torch.equal(_bits(q1), _bits(q_out)) and torch.equal(_bits(k1), _bits(m.k)) and torch.equal(_bits(v1), _bits(m.v))


def test_append_in_place_and_rows_of_a_single_call_or_many():
    m = RowsModel(n_q=8, n_kv=2, d=128, qk_norm=True)
    x = m.normal(50, 12 * 128)
    q = torch.empty(50, 8 * 128, dtype=torch.bfloat16, device=m.dev)
    m.append(0, [0, 20, 50], [2, 1], [5, 100], x, q)
    k0, v0 = m.k.clone(), m.v.clone()
    m.k[0].zero_(), m.v[0].zero_()
    y = x.clone()
    for i, (b, e, s, p) in enumerate([(0, 20, 2, 5), (20, 50, 1, 100)]):   # row after row, in place
        for r in range(b, e):
            m.append(0, [r, r + 1], [s], [p + r - b], y, y)
    m.status()
    assert torch.equal(_bits(y[:, : 8 * 128]), _bits(q)) and torch.equal(_bits(y[:, 8 * 128:]), _bits(x[:, 8 * 128:]))
    for s, a, b in ((2, 5, 25), (1, 100, 130)):
        assert torch.equal(_bits(m.k[0, s, :, a:b]), _bits(k0[0, s, :, a:b])) and torch.equal(_bits(m.v[0, s, :, a:b]), _bits(v0[0, s, :, a:b]))


ATTEND = [
    dict(n_q=4, n_kv=2, d=64, lens=[1], pos=[0], slots=None),                                    # one row, one key
    dict(n_q=8, n_kv=8, d=128, lens=[1, 1, 1], pos=[0, 63, 191], slots=[1, 2, 0]),
    dict(n_q=8, n_kv=1, d=128, lens=[1, 0, 1], pos=[64, 3, 128], slots=None),
    dict(n_q=16, n_kv=2, d=64, lens=[5, 3], pos=[187, 62], slots=[3, 1], first=2, behind=3),
    dict(n_q=8, n_kv=2, d=128, lens=[64], pos=[0], slots=None),
    dict(n_q=4, n_kv=4, d=64, lens=[65, 1, 130], pos=[0, 100, 61], slots=[2, 0, 3], behind=1),
    dict(n_q=16, n_kv=2, d=128, lens=[129, 17, 0, 1], pos=[40, 0, 0, 9], slots=None, page=8, pages=97),
    dict(n_q=8, n_kv=8, d=64, lens=[192, 33], pos=[0, 159], slots=[1, 0], page=16, pages=48, first=1),
    dict(n_q=2, n_kv=1, d=128, lens=[700], pos=[0], slots=None, max_seq=704, batch=1),
    dict(n_q=4, n_kv=1, d=64, lens=[300, 299], pos=[1500, 1001], slots=[1, 0], max_seq=1808, batch=2),
    dict(n_q=32, n_kv=8, d=128, lens=[1, 2], pos=[5000, 17], slots=None, max_seq=5056, batch=2, page=64, pages=160, layers=1),
    dict(n_q=8, n_kv=1, d=64, lens=[4], pos=[20003], slots=None, max_seq=20008, batch=1, layers=1),
    dict(n_q=32, n_kv=4, d=128, lens=[1, 40, 700, 8, 1, 256, 9, 1], pos=[1000, 0, 300, 500, 0, 0, 31, 1022], slots=[7, 6, 5, 4, 3, 2, 1, 0],
         max_seq=1024, batch=8, layers=1),
    dict(n_q=8, n_kv=1, d=128, lens=[1500], pos=[2500], slots=[0], max_seq=4000, batch=1, layers=1),
]


def _attend_case(case, pad=0, seed=0):
    c = dict(case)
    lens, pos, slots, first, behind = c.pop("lens"), c.pop("pos"), c.pop("slots"), c.pop("first", 0), c.pop("behind", 0)
    m = RowsModel(seed=seed, **c)
    begin = _begin(lens, first)
    q = m.normal(begin[-1] + behind, m.n_q * m.d + pad)
    return m, lens, pos, slots, begin, q


def _check_attend(m, layer, lens, pos, slots, begin, q, out, before=None):
    for i, (n, p) in enumerate(zip(lens, pos)):
        if not n:
            continue
        r, slot = slice(begin[i], begin[i + 1]), slots[i] if slots else i
        width = m.n_q * m.d
        want, bound = attend_exact(q[r, :width].view(n, m.n_q, m.d), m.cached(m.k, layer, slot, p + n), m.cached(m.v, layer, slot, p + n),
                                   torch.arange(p, p + n, device=m.dev))
        got = out[r, :width].view(n, m.n_q, m.d).double()
        assert torch.isfinite(got).all(), (i, n, p)
        far = ((got - want).abs() / bound).max()
        assert far <= 1, (i, n, p, float(far))
        if before is not None:
            before[r, :width] = out[r, :width]
    if before is not None:
        assert torch.equal(_bits(before), _bits(out))


@pytest.mark.parametrize("pad", [0, 40])
@pytest.mark.parametrize("case", ATTEND)
def test_attend(case, pad):
    m, lens, pos, slots, begin, q = _attend_case(case, pad)
    layer = m.layers - 1
    out = m.normal(q.shape[0], m.n_q * m.d + 8)
    before = out.clone()
    m.attend(layer, begin, slots, pos, q, out, workspace())
    m.status()
    _check_attend(m, layer, lens, pos, slots, begin, q, out, before)


def _random_case(seed):
    rng = random.Random(seed)
    n_kv, n = rng.choice([1, 2, 3, 8]), rng.choice([1, 2, 3, 7, 16])
    c = dict(n_kv=n_kv, n_q=n_kv * rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128]), batch=n, layers=1, page=rng.choice([0, 8, 16, 32, 64, 256]),
             first=rng.choice([0, 3]), behind=rng.choice([0, 5]))
    most = rng.choice([1, 4, 40, 300]) if n > 3 else rng.choice([1, 9, 130, 900])
    c["lens"] = [rng.choice([0, 1, rng.randint(0, most)]) for _ in range(n)]
    c["pos"] = [rng.choice([0, rng.randint(0, 200), rng.randint(0, 4000)]) for _ in range(n)]
    step = c["page"] or 1
    c["max_seq"] = -(-max(a + b for a, b in zip(c["lens"], c["pos"])) // step) * step or step
    if c["page"]:
        c["pages"] = n * c["max_seq"] // c["page"] + 3
    c["slots"] = rng.sample(range(n), n)
    return c


@pytest.mark.parametrize("seed", range(40))
def test_random_appends_and_attention(seed):
    case = _random_case(seed)
    m, lens, pos, slots, begin, _ = _attend_case(case, seed=seed)
    rows, width = begin[-1] + case["behind"], m.n_q * m.d
    x = m.normal(rows, (m.n_q + 2 * m.n_kv) * m.d)
    q, out, k0, v0 = m.normal(rows, width), m.normal(rows, width), m.k.clone(), m.v.clone()
    before, q_before = out.clone(), q.clone()
    m.append(0, begin, slots, pos, x, q)
    m.attend(0, begin, slots, pos, q, out, workspace())
    m.status()
    _check_attend(m, 0, lens, pos, slots, begin, q, out, before)
    written = 0
    for i, (n, p) in enumerate(zip(lens, pos)):
        r = slice(begin[i], begin[i + 1])
        q_before[r] = q[r]
        if n:
            at = torch.arange(p, p + n, device=m.dev)
            want, wk, _, size, ksize = append_exact(m, 0, at, x[r])
            noise = (m.d / 4 + 16) * F32_HALF
            assert ((q[r].view(n, m.n_q, m.d).double() - want).abs() <= BF16_HALF * want.abs() + noise * size).all()
            got = m.cached(m.k, 0, slots[i], p + n)[:, p:].transpose(0, 1).double()
            assert ((got - wk).abs() <= BF16_HALF * wk.abs() + noise * ksize).all()
            assert torch.equal(_bits(m.cached(m.v, 0, slots[i], p + n)[:, p:].transpose(0, 1)), _bits(x[r].view(n, -1, m.d)[:, m.n_q + m.n_kv:]))
            written += n * m.n_kv * m.d
    assert torch.equal(_bits(q_before), _bits(q))
    assert (_bits(m.k) != _bits(k0)).sum() <= written and (_bits(m.v) != _bits(v0)).sum() <= written


@pytest.mark.parametrize("scale", [0.0, 30.0])
def test_attend_flat_and_peaked_scores(scale):
    m, lens, pos, slots, begin, q = _attend_case(ATTEND[9])
    q *= scale
    out = torch.empty_like(q)
    m.attend(1, begin, slots, pos, q, out, workspace())
    m.status()
    _check_attend(m, 1, lens, pos, slots, begin, q, out)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("case", [ATTEND[i] for i in (1, 3, 5, 6, 9, 12)])
def test_cache_rows_above_a_position_never_reach_its_row(case, bad):
    """Rows behind a sequence's last hold `bad`; so does, in a second call, the sequence's last own row, which only it may see."""
    m, lens, pos, slots, begin, q = _attend_case(case)
    layer, out = m.layers - 1, torch.empty_like(q)
    rows = torch.arange(m.max_seq, device=m.dev)

    def put(i, first):   # into the sequence's rows first ..
        slot, cut = slots[i] if slots else i, rows >= first
        for cache in (m.k, m.v):
            if m.page:
                cache[layer][m.table[slot].long()[rows[cut] // m.page], :, rows[cut] % m.page] = bad
            else:
                cache[layer, slot, :, cut] = bad

    for i, (n, p) in enumerate(zip(lens, pos)):
        if n:
            put(i, p + n)
    m.attend(layer, begin, slots, pos, q, out, workspace())
    m.status()
    _check_attend(m, layer, lens, pos, slots, begin, q, out)
    first = out.clone()
    for i, (n, p) in enumerate(zip(lens, pos)):
        if n:
            put(i, p + n - 1)
    m.attend(layer, begin, slots, pos, q, out, workspace())
    m.status()
    for i, n in enumerate(lens):
        if n:
            a, b = begin[i], begin[i + 1]
            assert torch.equal(_bits(out[a:b - 1]), _bits(first[a:b - 1]))
            assert not torch.isfinite(out[b - 1, : m.n_q * m.d]).all()


def test_an_infinite_or_nan_value_reaches_the_rows_that_see_it():
    m, lens, pos, slots, begin, q = _attend_case(dict(n_q=8, n_kv=2, d=128, lens=[150], pos=[20], slots=[1]))
    m.v[0, 1, 0, 100, 3] = float("inf")
    m.v[0, 1, 1, 120, 70] = float("nan")
    out = torch.empty_like(q)
    m.attend(0, begin, slots, pos, q, out, workspace())
    m.status()
    o = out.view(150, 8, 128)
    want = torch.zeros(150, 8, 128, dtype=torch.bool, device=m.dev)
    want[80:, :4, 3] = True
    want[100:, 4:, 70] = True
    assert torch.equal(~torch.isfinite(o), want) and (o[80:, :4, 3] == float("inf")).all() and o[100:, 4:, 70].isnan().all()


@pytest.mark.parametrize("page", [0, 4096])
def test_a_cache_whose_offsets_pass_32_bits(page):
    """2^25 positions of 128 elements (smaller pages would be more of them than a decode step can hold).  All keys are zero but
    three, at the start, in the middle and at the end; their scores, 40, leave the others together less than 3.4e7 e^-40,
    2e-10, of the weight."""
    n, pos = (1 << 25) + 4096, (1 << 25) + 900
    pages = dict(page=page, pages=n // page) if page else {}
    m = RowsModel(n_q=2, n_kv=1, d=128, layers=1, batch=1, max_seq=n, fill=0.0, **pages)
    x = m.normal(3, 4 * 128)
    rotated, out = m.normal(3, 256), m.normal(3, 256)
    m.append(0, [0, 3], None, [pos], x, rotated)
    m.status()
    want, wk, _, size, ksize = append_exact(m, 0, torch.arange(pos, pos + 3, device=m.dev), x)
    noise = (128 / 4 + 16) * F32_HALF

    def row(cache, at):
        return cache[0, 0, 0, at] if not page else cache[0, int(m.table[0, at // page]), 0, at % page]

    assert ((rotated.view(3, 2, 128).double() - want).abs() <= BF16_HALF * want.abs() + noise * size).all()
    assert sum(int(torch.count_nonzero(c)) for c in m.v[0].split(1 << 14, 0)) <= 3 * 128
    for i in range(3):
        assert ((row(m.k, pos + i).double() - wk[i, 0]).abs() <= BF16_HALF * wk[i, 0].abs() + noise * ksize[i, 0]).all()
        assert torch.equal(_bits(row(m.v, pos + i)), _bits(x[i, 3 * 128:]))
        row(m.k, pos + i).zero_()
    queries = torch.zeros(3, 256, dtype=torch.bfloat16, device=m.dev)
    queries[:, 0] = queries[:, 128] = 64.0
    seen = [5, (1 << 24) + 77, pos + 1]
    for at in seen:
        row(m.k, at)[0] = 40 * 128 ** 0.5 / 64
        row(m.v, at).copy_(m.normal(128))
    m.attend(0, [0, 3], None, [pos], queries, out, workspace())
    m.status()
    for i in range(3):
        v = torch.stack([row(m.v, at) for at in seen if at <= pos + i]).double()
        # weights as they are rounded to bf16 against their sum, and the output once
        bound = 2 * BF16_HALF * v.abs().mean(0) + BF16_HALF * v.mean(0).abs() + 1e-6
        assert ((out[i].view(2, 128).double() - v.mean(0)).abs() <= bound).all()


def test_rows_far_apart():
    """Row strides of 2^31 elements of qkv, queries and outputs: the third row begins past 2^32."""
    stride = 1 << 31
    m = RowsModel(n_q=4, n_kv=2, d=64, layers=1, batch=1, max_seq=64)

    def spread(x):
        far = torch.empty(2 * stride + x.shape[1], dtype=torch.bfloat16, device=m.dev).as_strided(x.shape, (stride, 1))
        return far.copy_(x)

    x, work = m.normal(3, 8 * 64), workspace()
    near = torch.empty(3, 256, dtype=torch.bfloat16, device=m.dev), torch.empty(3, 256, dtype=torch.bfloat16, device=m.dev)
    far = spread(near[0]), spread(near[1])
    k0, v0, caches = m.k.clone(), m.v.clone(), []
    for rows, (q, out) in ((x, near), (spread(x), far)):
        m.k.copy_(k0)
        m.v.copy_(v0)
        m.append(0, [0, 3], None, [40], rows, q)
        m.attend(0, [0, 3], None, [40], q, out, work)
        m.status()
        caches.append((m.k.clone(), m.v.clone()))
    assert all(torch.equal(_bits(a), _bits(b)) for a, b in zip(near + caches[0], far + caches[1]))


def test_two_graphs_at_once():
    """Each on a stream of its own, with a workspace of its own."""
    case = dict(n_q=8, n_kv=2, d=128, batch=3, layers=1, max_seq=4096, page=0, lens=[1, 70, 3], pos=[4000, 1300, 9], slots=[0, 1, 2],
                first=0, behind=0)
    sides = []
    for seed in (1, 2):
        m, lens, pos, slots, begin, _ = _attend_case(case, seed=seed)
        q, logits = m.normal(begin[-1], m.n_q * m.d), m.normal(5, m.vocab, dtype=torch.float32)
        sides.append(SimpleNamespace(m=m, q=q, logits=logits, tokens=m.ints([3] * 5), work=workspace(), stream=torch.cuda.Stream(),
                                     lists=(m.ints(begin), m.ints(pos)), outs=[]))

    def run(s, stream):
        with torch.cuda.stream(stream):
            out, lp, ent = torch.empty_like(s.q), torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
            s.m.graph.rows_attend(0, 3, len(s.q), s.lists[0].data_ptr(), 0, s.lists[1].data_ptr(), s.q.data_ptr(), s.q.stride(0),
                                  out.data_ptr(), out.stride(0), s.work.data_ptr(), stream.cuda_stream)
            s.m.graph.rows_logprobs(5, s.logits.data_ptr(), M.ROWS_F32, s.m.vocab, s.tokens.data_ptr(), 0, lp.data_ptr(), ent.data_ptr(),
                                    0, 0, s.work.data_ptr(), stream.cuda_stream)
        return out, lp, ent

    alone = []
    for s in sides:
        alone.append(run(s, torch.cuda.current_stream()))
        s.m.status()
    for _ in range(20):
        for s in sides:
            s.outs.append(run(s, s.stream))
    for s, want in zip(sides, alone):
        s.m.status()
        for got in s.outs:
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_the_same_call_gives_the_same_bits_on_any_stream():
    m, lens, pos, slots, begin, q = _attend_case(ATTEND[12])
    first = torch.empty_like(q)
    m.attend(0, begin, slots, pos, q, first, workspace())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        out, work = torch.empty_like(q), workspace()
        side.wait_stream(torch.cuda.current_stream())
        m.attend(0, begin, slots, pos, q, out, work, stream=side.cuda_stream)
        side.synchronize()
        assert torch.equal(_bits(out), _bits(first))
    m.status()


def test_captured_calls_follow_the_lengths_of_each_replay():
    m = RowsModel(n_q=8, n_kv=2, d=64, max_seq=640, batch=3, layers=1, page=16, pages=140)
    rows = 256
    x, q, out = m.normal(rows, 12 * 64), torch.zeros(rows, 512, dtype=torch.bfloat16, device=m.dev), torch.zeros(rows, 512, dtype=torch.bfloat16, device=m.dev)
    begin, slots, pos, work = m.ints([0, 0, 0, 0]), m.ints([0, 1, 2]), m.ints([0, 0, 0]), workspace()

    def calls(stream):
        m.graph.rows_append(0, 3, rows, begin.data_ptr(), slots.data_ptr(), pos.data_ptr(), x.data_ptr(), M.ROWS_BF16, x.stride(0),
                            q.data_ptr(), q.stride(0), stream)
        m.graph.rows_attend(0, 3, rows, begin.data_ptr(), slots.data_ptr(), pos.data_ptr(), q.data_ptr(), q.stride(0), out.data_ptr(),
                            out.stride(0), work.data_ptr(), stream)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(torch.cuda.current_stream().cuda_stream)
    for lens, p, s in (([1, 1, 1], [300, 0, 77], [0, 1, 2]), ([200, 0, 56], [100, 600, 0], [2, 0, 1]), ([0, 0, 256], [0, 0, 384], [0, 1, 2]),
                       ([3, 2, 4], [16, 630, 333], [1, 2, 0]), ([0, 0, 0], [0, 0, 0], [0, 1, 2])):
        begin.copy_(m.ints(_begin(lens))), pos.copy_(m.ints(p)), slots.copy_(m.ints(s))
        k0, v0 = m.k.clone(), m.v.clone()
        out.fill_(7.0)
        graph.replay()
        m.status()
        got, k1 = out.clone(), m.k.clone()
        _check_attend(m, 0, lens, p, s, _begin(lens), q, got)
        assert (got[sum(lens):] == 7.0).all()
        m.k.copy_(k0), m.v.copy_(v0), out.fill_(7.0)
        calls(torch.cuda.current_stream().cuda_stream)
        m.status()
        assert torch.equal(_bits(out), _bits(got)) and torch.equal(_bits(m.k), _bits(k1))


# what the device finds: begin, slots, positions, the sequences left out, what the status says
WRONG = [
    ([0, 3, 2, 6], [0, 1, 2], [0, 0, 0], {0, 1, 2}, "row_begin.*sequence 1"),
    ([-1, 3, 4, 6], [0, 1, 2], [0, 0, 0], {0, 1, 2}, "row_begin.*sequence 0"),
    ([0, 3, 4, 7], [0, 1, 2], [0, 0, 0], {0, 1, 2}, "row_begin.*sequence 2"),
    ([0, 3, 4, 6], [0, 4, 2], [0, 0, 0], {1}, "sequence 1 has slot 4"),
    ([0, 3, 4, 6], [-1, 1, 2], [0, 0, 0], {0}, "sequence 0 has slot -1"),
    ([0, 3, 4, 6], [2, 1, 2], [0, 0, 50], {2}, "sequence 2 has slot 2"),
    ([0, 3, 4, 6], [0, 1, 2], [-1, 0, 0], {0}, "sequence 0 has position -1"),
    ([0, 3, 4, 6], [0, 1, 2], [0, 192, 0], {1}, "sequence 1 has position 192"),
    ([0, 3, 4, 6], [0, 1, 2], [0, 0, 191], {2}, "sequence 2 has position 192"),
    ([0, 3, 3, 6], [0, 0, 2], [0, 999, 0], set(), None),   # (a sequence without rows may say anything)
]


@pytest.mark.parametrize("begin,slots,pos,out_of,says", WRONG)
def test_wrong_sequences_are_reported_and_left_out(begin, slots, pos, out_of, says):
    m = RowsModel(n_q=8, n_kv=2, d=64)
    x, q, out = m.normal(6, 12 * 64), m.normal(6, 512), m.normal(6, 512)
    q0, out0, k0, v0 = q.clone(), out.clone(), m.k.clone(), m.v.clone()
    for call in (lambda: m.append(0, begin, slots, pos, x, q), lambda: m.attend(0, begin, slots, pos, q, out, workspace())):
        call()
        if says is None:
            m.status()
        else:
            with pytest.raises(M.MpkError, match=says) as e:
                m.status()
            assert e.value.status == M.MPK_ERR_DEVICE
            m.graph.reset()
    m.status()
    for i in range(3):
        r = slice(max(begin[i], 0), max(begin[i + 1], 0))
        same = torch.equal(_bits(q[r]), _bits(q0[r])) and torch.equal(_bits(out[r]), _bits(out0[r]))
        assert same == (i in out_of or begin[i] == begin[i + 1]), i
    for s in range(4):
        touched = any(s == slots[i] and i not in out_of and begin[i + 1] > begin[i] for i in range(3))
        assert torch.equal(_bits(m.k[0, s]), _bits(k0[0, s])) != touched and torch.equal(_bits(m.v[0, s]), _bits(v0[0, s])) != touched
    assert torch.equal(_bits(m.k[1]), _bits(k0[1])) and torch.equal(_bits(m.v[1]), _bits(v0[1]))


@pytest.mark.parametrize("bad", [-1, 50, 2 ** 31 - 1])
@pytest.mark.parametrize("lens", [[1, 1], [2, 40]])
def test_a_page_outside_the_pool_is_reported_and_never_dereferenced(bad, lens):
    m = RowsModel(n_q=8, n_kv=2, d=64, page=16, pages=50)
    m.table[1, 2] = bad
    begin, rows = _begin(lens), sum(lens)
    x, q, out = m.normal(rows, 12 * 64), torch.zeros(rows, 512, dtype=torch.bfloat16, device=m.dev), m.normal(rows, 512)
    k0 = m.k.clone()
    for call in (lambda: m.append(0, begin, None, [10, 33], x, q), lambda: m.attend(0, begin, None, [10, 33], q, out, workspace())):
        call()
        with pytest.raises(M.MpkError, match="sequence 1: a page-table entry") as e:
            m.status()
        assert e.value.status == M.MPK_ERR_DEVICE
        m.graph.reset()
    _check_attend(m, 0, lens[:1], [10], None, begin, q, out)   # (the other sequence has its results)
    mine = {int(p) for p in torch.cat([m.table[0], m.table[1]]).tolist() if 0 <= p < 50}
    others = torch.tensor([p for p in range(50) if p not in mine], device=m.dev)
    assert torch.equal(_bits(m.k[0][others]), _bits(k0[0][others]))


def test_a_paged_graph_without_a_table_is_refused():
    m = RowsModel(n_q=8, n_kv=2, d=64, page=16, pages=50)
    g = M.compile_graph(m.shape, {**{n: t.data_ptr() for n, t in m.outer.items()}, "layers": [{n: t.data_ptr() for n, t in w.items()} for w in m.w]},
                        (m.k.data_ptr(), m.v.data_ptr()), fusion=31, kv_page_size=16, kv_pages=50)
    x, b = m.normal(1, 768), m.ints([0, 1])
    with pytest.raises(M.MpkError, match="page table"):
        g.rows_append(0, 1, 1, b.data_ptr(), 0, b.data_ptr(), x.data_ptr(), 0, 768, x.data_ptr(), 768)
    with pytest.raises(M.MpkError, match="page table"):
        g.rows_attend(0, 1, 1, b.data_ptr(), 0, b.data_ptr(), x.data_ptr(), 768, workspace().data_ptr(), 512, workspace().data_ptr())


# ---------------------------------------------------------------------------------- together
def _layer_rest(m, w, h, o):
    h = h + o.float() @ w["wo"].float().t()
    y = _rms(m, h, w["mlp_norm"])
    g, u = (y @ w["wgu"].float().t()).chunk(2, -1)
    return h + (torch.nn.functional.silu(g) * u) @ w["wd"].float().t()


def _rms(m, x, g):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + m.eps) * g.float()


@pytest.mark.parametrize("kw", [dict(n_q=8, n_kv=2, d=64, qk_norm=True), dict(n_q=8, n_kv=2, d=128, page=16, pages=60, theta=1e6)])
def test_prompts_through_rows_then_decoding_equals_token_by_token(kw):
    """Prompts of three sequences through the layers with the row calls, in two chunks; the last rows' logits scored; then
    two decode steps of the graph on the cache they left: against the graph fed token by token."""
    kw = dict(kw, batch=3, vocab=512, layers=3, max_seq=192)
    a, b = RowsModel(seed=5, fill=float("nan"), **kw), RowsModel(seed=5, fill=float("nan"), **kw)
    rng = torch.Generator().manual_seed(3)
    lens = [37, 5, 70]
    prompts = [torch.randint(512, (n,), generator=rng, dtype=torch.int32) for n in lens]
    # token by token: a sequence that has ended feeds its last token again (the same row, written again)
    logits = torch.zeros(3, 512, device="cuda")
    for t in range(max(lens)):
        at = [min(t, n - 1) for n in lens]
        tok, pos = a.ints([int(p[i]) for p, i in zip(prompts, at)]), a.ints(at)
        a.graph.decode_step(tok.data_ptr(), pos.data_ptr(), logits.data_ptr(), torch.cuda.current_stream().cuda_stream)
    a.status()
    want = logits.clone()
    work, done = workspace(), [0, 0, 0]
    for size in (33, 64):
        now = [min(size, n - d) for n, d in zip(lens, done)]
        begin = _begin(now)
        tokens = torch.cat([p[d:d + n] for p, d, n in zip(prompts, done, now)]).cuda().long()
        h = b.outer["embed"][tokens].float()
        for l, w in enumerate(b.w):
            qkv = _rms(b, h, w["attn_norm"]) @ w["wqkv"].float().t()
            q, o = (torch.empty(len(tokens), b.n_q * b.d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            b.append(l, begin, None, done, qkv, q)
            b.attend(l, begin, None, done, q, o, work)
            h = _layer_rest(b, w, h, o)
        for i, n in enumerate(now):
            if n:
                logits[i] = _rms(b, h[begin[i + 1] - 1], b.outer["final_norm"]) @ b.outer["lm_head"].float().t()
        done = [d + n for d, n in zip(done, now)]
    b.status()
    # queries, probabilities and outputs of three layers in bf16: the decoder's are fp32
    scale = want.abs().max()
    assert (logits - want).abs().max() < 8 * BF16_HALF * scale
    tok = want.argmax(-1).to(torch.int32)
    lp, ent = torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    ids, tops = torch.empty(3, 4, dtype=torch.int32, device="cuda"), torch.empty(3, 4, device="cuda")
    pos = b.ints(lens)
    for _ in range(2):
        out = []
        for m in (a, b):
            lg = torch.empty(3, 512, device="cuda")
            m.graph.decode_step(tok.data_ptr(), pos.data_ptr(), lg.data_ptr(), torch.cuda.current_stream().cuda_stream)
            m.status()
            out.append(lg)
        assert torch.isfinite(out[1]).all() and (out[0] - out[1]).abs().max() < 8 * BF16_HALF * scale
        tok = out[0].argmax(-1).to(torch.int32)
        b.graph.rows_logprobs(3, out[0].data_ptr(), M.ROWS_F32, 512, tok.data_ptr(), 4, lp.data_ptr(), ent.data_ptr(), ids.data_ptr(),
                              tops.data_ptr(), work.data_ptr(), torch.cuda.current_stream().cuda_stream)
        b.status()
        p = torch.log_softmax(out[0].double(), -1)
        assert torch.equal(ids[:, 0], tok) and (lp - p.amax(-1)).abs().max() < 1e-5 and torch.equal(lp, tops[:, 0])
        assert (ent + (p.exp() * p).sum(-1)).abs().max() < 1e-4
        pos = pos + 1


def test_calls_on_the_graphs_of_a_set_share_its_cache():
    from types import SimpleNamespace
    m = RowsModel(n_q=8, n_kv=2, d=64, batch=4, layers=2)
    ptrs = {n: t.data_ptr() for n, t in m.outer.items()}
    ptrs["layers"] = [{n: t.data_ptr() for n, t in w.items()} for w in m.w]
    s = M.compile_set(SimpleNamespace(**vars(m.shape)), ptrs, (m.k.data_ptr(), m.v.data_ptr()), fusion=31, transitive_reduction=1)
    x = m.normal(9, 12 * 64)
    for i in range(len(s)):
        outs = []
        for g in (m.graph, s.graph(i)):
            m.k.zero_(), m.v.zero_()
            q, o = (torch.empty(9, 512, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            b, p = m.ints([0, 9]), m.ints([30])
            g.rows_append(1, 1, 9, b.data_ptr(), 0, p.data_ptr(), x.data_ptr(), 0, 768, q.data_ptr(), 512)
            g.rows_attend(1, 1, 9, b.data_ptr(), 0, p.data_ptr(), q.data_ptr(), 512, o.data_ptr(), 512, workspace().data_ptr())
            torch.cuda.synchronize()
            g.status()
            outs.append((q, o, m.k.clone(), m.v.clone()))
        assert all(torch.equal(_bits(u), _bits(w)) for u, w in zip(*outs))
    s.destroy()


@pytest.mark.parametrize("kw", [dict(n_q=8, n_kv=2, d=128, qk_norm=True), dict(n_q=16, n_kv=2, d=64, page=16, pages=260), dict(n_q=3, n_kv=3, d=64)])
@pytest.mark.parametrize("lens", [[20, 0, 7], [300, 1, 211], [3, 500, 430]])
def test_many_rows_in_place(lens, kw):
    """Up to and above 512 rows, a wavefront has other groups of heads: the same bits as with the queries in a place of their own."""
    m = RowsModel(batch=3, max_seq=1024, **kw)
    pos, slots, begin, width = [500, 3, 17], [1, 2, 0], _begin(lens, 2), m.n_q * m.d
    x = m.normal(begin[-1] + 3, (m.n_q + 2 * m.n_kv) * m.d + 16)
    q = x[:, :width].clone()
    k0, v0, y = m.k.clone(), m.v.clone(), x.clone()
    m.append(1, begin, slots, pos, x, q)
    m.status()
    k1, v1 = m.k.clone(), m.v.clone()
    m.k.copy_(k0), m.v.copy_(v0)
    m.append(1, begin, slots, pos, y, y)
    m.status()
    assert torch.equal(_bits(y[:, :width]), _bits(q)) and torch.equal(_bits(y[:, width:]), _bits(x[:, width:]))
    assert torch.equal(_bits(m.k), _bits(k1)) and torch.equal(_bits(m.v), _bits(v1)) and not torch.equal(_bits(k1), _bits(k0))


# More runs of a tile than a wavefront of the join has lanes (144, 214, 137, and 167 of one row in a call with rows to spare, twice as
# long as they would be for the runs to be no more than the join holds); more units than run at once, tiles of several sequences (520,
# 544) and single rows of many heads (768 and 1152, a workgroup takes several).
MANY = [
    dict(n_q=1, n_kv=1, d=64, lens=[129], pos=[64000], slots=None, max_seq=64192, batch=1, layers=1),
    dict(n_q=1, n_kv=1, d=64, lens=[129], pos=[150000], slots=None, max_seq=150200, batch=1, layers=1),
    dict(n_q=2, n_kv=1, d=128, lens=[129], pos=[96000], slots=None, max_seq=96192, batch=1, layers=1, page=64, pages=1503),
    dict(n_q=1, n_kv=1, d=64, lens=[1], pos=[64000], slots=None, max_seq=64192, batch=1, layers=1, behind=199),
    dict(n_q=8, n_kv=8, d=128, lens=[1100, 1, 700, 300, 0, 900, 64, 1300], pos=[5, 3000, 1700, 0, 9, 40, 2900, 2600], slots=[3, 1, 0, 2, 7, 6, 5, 4],
         max_seq=4000, batch=8, layers=1),
    dict(n_q=16, n_kv=8, d=64, lens=[600, 1, 350, 150, 0, 450, 32, 650], pos=[5, 3000, 1700, 0, 9, 40, 2900, 2600], slots=None, max_seq=4000,
         batch=8, layers=1, page=16, pages=2003),
    dict(n_q=32, n_kv=32, d=128, lens=[1] * 16, pos=[256 * (7 * i % 16 + 1) for i in range(16)], slots=None, max_seq=4200, batch=16, layers=1),
    dict(n_q=48, n_kv=48, d=64, lens=[1] * 16, pos=[256 * (7 * i % 16 + 1) for i in range(16)], slots=None, max_seq=4200, batch=16, layers=1),
]


@pytest.mark.parametrize("case", MANY)
def test_attend_many_runs_and_units(case):
    m, lens, pos, slots, begin, q = _attend_case(case)
    out = m.normal(q.shape[0], m.n_q * m.d)
    before = out.clone()
    m.attend(0, begin, slots, pos, q, out, workspace())
    m.status()
    _check_attend(m, 0, lens, pos, slots, begin, q, out, before)


def test_a_call_of_no_rows_does_nothing():
    """Not even a workspace or a buffer is needed, and the sequences may say anything but NULL."""
    m = RowsModel(n_q=8, n_kv=2, d=64)
    k0, v0, lists = m.k.clone(), m.v.clone(), m.ints([0, 0, 0])
    m.graph.rows_append(1, 2, 0, lists.data_ptr(), 0, lists.data_ptr(), 0, M.ROWS_F32, 0, 0, 0)
    m.graph.rows_attend(1, 2, 0, lists.data_ptr(), 0, lists.data_ptr(), 0, 0, 0, 0, 0)
    m.graph.rows_logprobs(0, 0, M.ROWS_F32, 0, 0, 4, 0, 0, 0, 0, 0)
    m.status()
    assert torch.equal(_bits(m.k), _bits(k0)) and torch.equal(_bits(m.v), _bits(v0))


def test_two_graphs_at_once_cut_their_rows():
    """Rows of logits in runs, joined through each graph's own counters and each call's own workspace."""
    rows, vocab, k = 6, 150011, 20
    sides = []
    for seed in (1, 2):
        m = RowsModel(n_q=4, n_kv=2, d=64, batch=1, layers=1, max_seq=64, vocab=vocab, seed=seed)
        x = m.normal(rows, vocab, dtype=torch.float32)
        sides.append(SimpleNamespace(m=m, x=x, tokens=m.ints([7 * seed] * rows), work=workspace(), stream=torch.cuda.Stream(), outs=[]))

    def run(s, stream):
        with torch.cuda.stream(stream):
            lp, ent = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
            ids, tops = torch.empty(rows, k, dtype=torch.int32, device="cuda"), torch.empty(rows, k, device="cuda")
            s.m.graph.rows_logprobs(rows, s.x.data_ptr(), M.ROWS_F32, vocab, s.tokens.data_ptr(), k, lp.data_ptr(), ent.data_ptr(), ids.data_ptr(),
                                    tops.data_ptr(), s.work.data_ptr(), stream.cuda_stream)
        return lp, ent, ids, tops

    alone = []
    for s in sides:
        alone.append(run(s, torch.cuda.current_stream()))
        s.m.status()
        best = s.x.double().sort(dim=-1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(alone[-1][2].long(), best)
    for _ in range(30):
        for s in sides:
            s.outs.append(run(s, s.stream))
    for s, want in zip(sides, alone):
        s.m.status()
        for got in s.outs:
            assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("case", [ATTEND[i] for i in (3, 5, 6, 9, 10)])
def test_a_query_that_is_not_finite_reaches_its_own_row_and_head_alone(case, bad):
    m, lens, pos, slots, begin, q = _attend_case(case)
    out, poisoned = torch.empty_like(q), torch.empty_like(q)
    m.attend(m.layers - 1, begin, slots, pos, q, out, workspace())
    m.status()
    hit = torch.zeros(q.shape[0], m.n_q, dtype=torch.bool, device=m.dev)
    for i, n in enumerate(lens):
        for t in range(0, n, 7):
            hit[begin[i] + t, (3 * t + i) % m.n_q] = True
    q.view(-1, m.n_q, m.d)[..., 5].masked_fill_(hit, bad)
    m.attend(m.layers - 1, begin, slots, pos, q, poisoned, workspace())
    m.status()
    a, b = out.view(-1, m.n_q, m.d), poisoned.view(-1, m.n_q, m.d)
    for i, n in enumerate(lens):
        r = slice(begin[i], begin[i] + n)
        clean = ~hit[r]
        assert torch.equal(_bits(a[r][clean]), _bits(b[r][clean]))
        assert b[r][hit[r]].isnan().all()   # (infinite scores have no softmax)
