"""mpk_tree_verify on the GPU against the definition in 64 bits."""
import math
import random
from fractions import Fraction

import pytest
import torch

import paper_2512_22219_amd as M
from tests.tree_util import F32_HALF, TreeModel, tree, verify_exact, workspace

pytestmark = pytest.mark.gpu


def _begin(lens, first=0):
    out = [first]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _tokens(gen, logits, parents, begin, draft, once, temperatures):
    """Tokens that the walk has something to do with: near the top of the parent's row, or drawn from the draft's."""
    tokens = [0] * logits.shape[0]
    for i in range(len(begin) - 1):
        seen = {}
        for t in range(begin[i], begin[i + 1]):
            p = parents[t]
            if p < 0:
                continue
            row = begin[i] + p
            j = seen[p] = seen.get(p, -1) + 1
            if draft is not None:
                q = draft[row].double().clone()
                for u in range(begin[i], t):
                    if once and parents[u] == p:
                        q[tokens[u]] = 0
                tokens[t] = int(torch.multinomial(q, 1, generator=gen)) if q.sum() > 0 else 0
            else:
                tokens[t] = int(logits[row].float().nan_to_num(-1e30).topk(min(j + 1, logits.shape[1])).indices[-1])
    return tokens


def _check(m, begin, parents, tokens, logits, out, temperatures, uniforms, draft=None, once=False, work=None):
    lengths, path, nxt, lp = (t.cpu() for t in out)
    mine = torch.zeros(len(path), dtype=torch.bool)
    for i in range(len(begin) - 1):
        r = slice(begin[i], begin[i + 1])
        mine[r] = True
        if begin[i] == begin[i + 1]:
            assert int(lengths[i]) == 0 and int(nxt[i]) == -1
            continue
        walk, token, logs = verify_exact(parents[r], tokens[r], logits[r], temperatures[i] if temperatures is not None else 0.0,
                                         [0.0] * (r.stop - r.start) if uniforms is None else uniforms[r].tolist(), None if draft is None else draft[r], once)
        rest = r.stop - r.start - len(walk)
        assert int(lengths[i]) == len(walk) and path[r].tolist() == walk + [-1] * rest and int(nxt[i]) == token, i
        want = torch.tensor(logs + [0.0] * rest, dtype=torch.float64)
        # 64-bit sums to 1e-9 or better, one rounding to 32 bits
        far = (lp[r].double() - want).abs() - (F32_HALF * want.abs() + 2e-9)
        assert (torch.isnan(want) == torch.isnan(lp[r])).all() and not (far > 0).any(), (i, float(far.max()))
    assert (path[~mine] == 77).all() and (lp[~mine] == 77).all()


def _case(seed, vocab, lens, kinds, dtype=torch.float32, draft=None, temperatures=None, first=0, behind=0, pad=0, std=2.0, batch=16, masked=0.0, calls=1, **opts):
    gen = torch.Generator().manual_seed(seed)
    m = TreeModel(n_q=2, n_kv=1, batch=batch, max_seq=8, vocab=vocab, layers=1, **opts)
    begin = _begin(lens, first)
    rows = begin[-1] + behind
    parents = [55] * first + sum((tree(n, k, seed + i) for i, (n, k) in enumerate(zip(lens, kinds))), []) + [-55] * behind
    x = torch.randn(rows, vocab, generator=gen) * std
    up = torch.randint(vocab, (rows,), generator=gen)
    x[torch.arange(rows), up] += 8 * torch.rand(rows, generator=gen)
    if masked:
        gone = torch.rand(rows, vocab, generator=gen) < masked
        gone[torch.arange(rows), up] = False
        x[gone] = -math.inf
    logits = x.to(dtype)
    q = None
    if draft:
        q = torch.softmax((logits.float() + torch.randn(rows, vocab, generator=gen)) / 1.2, 1)
    once = draft == "once"
    tokens = _tokens(gen, logits, parents, begin, q, once, temperatures)
    uniforms = torch.rand(rows, generator=gen)
    if temperatures is None:
        temps = None
    else:
        temps = [temperatures[i % len(temperatures)] for i in range(len(lens))]
    dev = torch.device("cuda")
    wide = torch.full((rows, vocab + pad), float("nan"), dtype=dtype, device=dev)
    wide[:, :vocab] = logits.to(dev)
    dwide = None
    if q is not None:
        dwide = torch.full((rows, vocab + pad), float("nan"), device=dev)
        dwide[:, :vocab] = q.to(dev)
    for _ in range(calls):
        out = m.verify(begin, parents, tokens, wide, workspace(), draft=dwide, once=once, temperatures=temps, uniforms=None if temps is None else uniforms)
        m.status()
        _check(m, begin, parents, tokens, logits, out, temps, uniforms, q, once)
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("draft", [None, "drawn", "once"])
@pytest.mark.parametrize("vocab,pad", [(1, 0), (2, 1), (63, 0), (64, 3), (257, 0), (1000, 8), (4097, 1), (33001, 7)])
def test_verify(vocab, pad, draft, dtype):
    _case(vocab, vocab, [1, 0, 2, 9, 40, 17, 5, 6], ["chain", "chain", "chain", "star", "random", "two", "star", "chain"], dtype, draft,
          [1.0, 0.6, 0.0, 1.3, 1.0, 0.9, 1.7, 1.0], first=2, behind=1, pad=pad)


@pytest.mark.parametrize("draft", [None, "drawn", "once"])
@pytest.mark.parametrize("temperatures", [None, [0.0], [1.0], [0.25, 4.0]])
def test_verify_at_a_large_vocabulary(draft, temperatures):
    _case(3, 151936, [8, 1, 5], ["random", "chain", "star"], torch.bfloat16, draft, temperatures)


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("draft", [None, "drawn", "once"])
def test_workgroups_that_are_late(draft, seed):
    """Every workgroup waits at random, in each round, up to twice as long as the others wait for it: the same tokens."""
    for dtype in (torch.float32, torch.bfloat16):
        _case(seed, 70001, [9, 1, 30], ["chain", "chain", "random"], dtype, draft, [1.0, 0.0, 0.8], debug_flags=M.DEBUG_JITTER)


@pytest.mark.parametrize("draft", [None, "drawn", "once"])
@pytest.mark.parametrize("vocab,lens,dtype", [(100003, [3, 9, 1, 0, 6, 2, 4, 5, 1, 7, 3, 3, 2, 8, 1, 5], torch.bfloat16),
                                              (100003, [3, 9, 1, 0, 6, 2, 4, 5, 1, 7, 3, 3, 2, 8, 1, 5], torch.float32),
                                              (262144, [6, 3], torch.float32), (262145, [6], torch.bfloat16), (600001, [5], torch.float32)])
def test_verify_rows_of_several_steps_a_workgroup(vocab, lens, dtype, draft):
    """More logits than a workgroup takes at once: many sequences, or more than the largest number of chunks."""
    kinds = [("chain", "star", "random")[i % 3] for i in range(len(lens))]
    _case(vocab + len(lens), vocab, lens, kinds, dtype, draft, [1.0, 0.0, 0.7], pad=1)


@pytest.mark.parametrize("draft", [None, "drawn"])
def test_many_workgroups_that_are_late_on_one_graph(draft):
    """As above with every sequence a call can have, call after call on one graph: words of earlier rounds are there, and start over."""
    _case(1, 40001, [5, 1, 7, 3, 0, 9, 2, 4, 6, 1, 3, 8, 2, 5, 7, 4], ["random"] * 16, torch.float32, draft, [1.0, 0.0, 0.8], calls=8, debug_flags=M.DEBUG_JITTER)


@pytest.mark.parametrize("draft", [None, "once"])
@pytest.mark.parametrize("kind", ["chain", "star", "random"])
def test_verify_the_largest_trees(kind, draft):
    _case(7, 300, [256, 255, 1], [kind] * 3, torch.float32, draft, [1.0, 0.0, 1.0])


@pytest.mark.parametrize("draft", [None, "drawn"])
@pytest.mark.parametrize("std", [0.0, 0.01, 30.0, 3000.0, 1e30])
def test_verify_flat_and_peaked_rows(std, draft):
    _case(11, 5000, [6, 20, 3], ["chain", "random", "star"], torch.float32, draft, [1.0, 0.5, 2.0], std=std)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("masked", [0.5, 0.999, 1.0])
def test_verify_under_a_grammar(masked, dtype):
    """Most tokens, or all but one, are ruled out."""
    out = _case(5, 3001, [6, 20, 3, 9], ["chain", "random", "star", "two"], dtype, None, [1.0, 0.5, 0.0, 1.0], masked=masked)
    assert (out[2] >= 0).all()


@pytest.mark.parametrize("seed", range(40))
def test_random_verifications(seed):
    rng = random.Random(seed)
    n = rng.choice([1, 2, 5, 16])
    lens = [rng.choice([0, 1, rng.randint(1, 10), rng.randint(1, 60)]) for _ in range(n)]
    _case(seed, rng.choice([17, 128, 999, 4096, 20011]), lens, [rng.choice(["chain", "star", "two", "random"]) for _ in lens],
          rng.choice([torch.float32, torch.bfloat16]), rng.choice([None, None, "drawn", "once"]), rng.choice([None, [0.0, 1.0], [1.0], [0.7, 1.1]]),
          first=rng.choice([0, 1]), behind=rng.choice([0, 4]), pad=rng.choice([0, 0, 1, 5, 8]), masked=rng.choice([0.0, 0.0, 0.8]))


@pytest.mark.parametrize("draft", [None, "drawn", "once"])
def test_the_tokens_have_the_targets_distribution(draft):
    """The first two tokens behind the root, over many uniform numbers, against p(a) p(b | a): trees over a vocabulary of four, where
    a tree holds every token's continuation, so that p(b | a) is the same whichever way a came about."""
    V, S, calls, temp = 4, 16, 120, 0.8
    m = TreeModel(n_q=2, n_kv=1, batch=S, max_seq=8, vocab=V, layers=1)
    gen = torch.Generator().manual_seed(9)
    logit_of = torch.randn(V, V, generator=gen) * 1.5       # row: the token in front
    root_logits, guess = torch.randn(V, generator=gen) * 1.5, torch.randn(V + 1, V, generator=gen)
    q_root, q_of = torch.softmax(guess[V], 0), torch.softmax(guess[:V], 1)
    work, counts, drawn_gen = workspace(), torch.zeros(V, V), torch.Generator().manual_seed(10)
    for _ in range(calls):
        parents, tokens, rows, qs = [], [], [], []
        for _ in range(S):
            # three children of the root (chosen: 2, 0, 2 again), two of each of these
            if draft is None:
                first, second = [2, 0, 2], lambda a: [1, 3]  # noqa: E731
            else:
                first = torch.multinomial(q_root, 3, replacement=draft == "drawn", generator=drawn_gen).tolist()
                second = lambda a: torch.multinomial(q_of[a], 2, replacement=draft == "drawn", generator=drawn_gen).tolist()  # noqa: E731
            parents += [-1, 0, 0, 0] + [1, 1, 2, 2, 3, 3]
            below = [x for a in first for x in second(a)]
            tokens += [0] + first + below
            rows += [root_logits] + [logit_of[a] for a in first + below]
            qs += [q_root] + [q_of[a] for a in first + below]
        n = len(parents)
        logits, u = torch.stack(rows).cuda(), torch.rand(n, generator=gen)
        lengths, path, nxt, _ = (t.cpu() for t in m.verify(list(range(0, n + 1, 10)), parents, tokens, logits, work, torch.stack(qs).cuda() if draft else None,
                                                             draft == "once", [temp] * S, u))
        for i in range(S):
            walk = [tokens[10 * i + t] for t in path[10 * i:10 * i + int(lengths[i])].tolist()[1:]] + [int(nxt[i])]
            if len(walk) == 1:   # the token behind it is drawn as ever
                walk.append(int(torch.multinomial(torch.softmax(logit_of[walk[0]] / temp, 0), 1, generator=gen)))
            counts[walk[0], walk[1]] += 1
    m.status()
    p = torch.softmax(root_logits / temp, 0)[:, None] * torch.softmax(logit_of / temp, 1)
    total = S * calls
    # a count is binomial: five standard deviations, and one for the smallest
    assert ((counts - total * p).abs() <= 5 * (total * p * (1 - p)).sqrt() + 1).all(), (counts, total * p)


def test_numbers_on_the_edge():
    """u = 0 accepts whatever has any probability and draws the first token that has; the largest number below 1 draws the last."""
    V = 700
    m = TreeModel(n_q=2, n_kv=1, batch=16, max_seq=8, vocab=V, layers=1)
    x = torch.full((6, V), -math.inf)
    x[:, 5:650] = 0.0
    x[0, 9] = -200.0
    work, below_one = workspace(), 1 - 2 ** -24
    parents, tokens = [-1, 0, 1, -1, 0, 1], [0, 9, 4, 0, 700, 9]
    for u, want in (([0.0, 0.0, 0.0], [2, 2, 5]), ([below_one, 0.0, 0.0], [2, 2, 649]), ([below_one, 1e-3, 0.0], [1, 1, 649])):
        out = m.verify([0, 3], parents[:3], tokens[:3], x[:3].cuda(), work, temperatures=[1.0], uniforms=u)
        m.status()
        # node 1 (token 9: e^-200) is accepted at u = 0 alone, node 2 (token 4: ruled out) never
        assert [int(out[0][0]), len([t for t in out[1].tolist() if t >= 0]), int(out[2][0])] == want


def test_rows_without_a_distribution_end_the_walk():
    V = 1000
    m = TreeModel(n_q=2, n_kv=1, batch=16, max_seq=8, vocab=V, layers=1)
    work = workspace()
    for dtype in (torch.float32, torch.bfloat16):
        for bad in (math.nan, math.inf, None):
            x = torch.randn(8, V)
            x[0, 7] = 40.0
            if bad is None:
                x[1] = -math.inf
            else:
                x[1, 999] = bad
            x[5, 0] = math.nan   # (a node that the walk does not come to)
            for temp in (0.0, 1.0):
                out = m.verify([0, 4, 8], [-1, 0, 1, 2, -1, 0, 0, 0], [0, 7, 1, 1, 0, 1, 2, 3], x.to(dtype).cuda(), work, temperatures=[temp, 0.0],
                               uniforms=[0.5] * 8)
                m.status()
                assert out[0].tolist()[0] == 2 and out[1].tolist()[:4] == [0, 1, -1, -1] and int(out[2][0]) == -1
                lp = out[3].tolist()
                assert math.isfinite(lp[0]) and math.isnan(lp[1]) and lp[2:4] == [0.0, 0.0] and int(out[2][1]) >= 0


def test_a_draft_that_knows_no_other_token():
    """Draft and target agree on one token, the draft's only one; and a draft whose tokens are all drawn: nothing is left to subtract."""
    V = 64
    m = TreeModel(n_q=2, n_kv=1, batch=16, max_seq=8, vocab=V, layers=1)
    x, q, work = torch.full((4, V), -math.inf), torch.zeros(4, V), workspace()
    x[:, 3], q[:, 3] = 0.0, 1.0
    out = m.verify([0, 4], [-1, 0, 1, 2], [0, 3, 3, 3], x.cuda(), work, q.cuda(), True, [1.0], [0.9] * 4)
    assert out[0].tolist() == [4] and out[2].tolist() == [3]
    y = torch.zeros(4, V)
    y[:, 3] = -5.0
    for once in (False, True):   # token 3 is refused, its twins have no draft distribution left (once)
        out = m.verify([0, 4], [-1, 0, 0, 0], [0, 3, 3, 3], y.cuda(), work, q.cuda(), once, [1.0], [0.5] * 4)
        m.status()
        path, token, _ = verify_exact([-1, 0, 0, 0], [0, 3, 3, 3], y, 1.0, [0.5] * 4, q, once)
        assert out[0].tolist() == [1] and path == [0] and out[2].tolist() == [token]


WRONG = [
    (dict(begin=[0, 3, 2, 6]), {0, 1, 2}, "row_begin.*sequence 1"), (dict(begin=[0, 3, 4, 7]), {0, 1, 2}, "row_begin.*sequence 2"),
    (dict(parents=[0, 0, 0, -1, -1, 0]), {0}, "sequence 0: node 0"), (dict(parents=[-1, 0, 2, -1, -1, 0]), {0}, "sequence 0: node 2"),
    (dict(parents=[-1, 0, -1, -1, -1, 0]), {0}, "sequence 0: node 2"), (dict(parents=[-1, 0, 0, -1, -1, -2]), {2}, "sequence 2: node 1"),
    (dict(temperatures=[1.0, -1.0, 1.0]), {1}, "sequence 1 has the temperature -1"), (dict(temperatures=[1.0, 1.0, math.nan]), {2}, "sequence 2 has the temperature"),
    (dict(temperatures=[math.inf, 1.0, 1.0]), {0}, "sequence 0 has the temperature inf"),
]


@pytest.mark.parametrize("change,left,says", WRONG)
def test_wrong_sequences_are_reported_and_left_out(change, left, says):
    V = 300
    m = TreeModel(n_q=2, n_kv=1, batch=4, max_seq=8, vocab=V, layers=1)
    args = dict(dict(begin=[0, 3, 4, 6], parents=[-1, 0, 0, -1, -1, 0], temperatures=[1.0, 1.0, 1.0]), **change)
    x = torch.randn(6, V)
    out = m.verify(args["begin"], args["parents"], [1, 2, 3, 4, 5, 6], x.cuda(), workspace(), temperatures=args["temperatures"], uniforms=[0.3] * 6)
    with pytest.raises(M.MpkError, match=says) as e:
        m.status()
    assert e.value.status == M.MPK_ERR_DEVICE
    m.graph.reset()
    all_out = "row_begin" in says
    for i in range(3):
        r = slice(args["begin"][i], args["begin"][i + 1])
        if i in left:
            assert int(out[0][i]) == 0 and int(out[2][i]) == -1
            if not all_out:
                assert (out[1][r] == -1).all() and (out[3][r] == 0).all()
        else:
            path, token, _ = verify_exact(args["parents"][r], [1, 2, 3, 4, 5, 6][r], x[r], 1.0, [0.3] * 6)
            assert int(out[0][i]) == len(path) and int(out[2][i]) == token
    if all_out:
        assert (out[1] == 77).all() and (out[3] == 77).all()
    # and the next call on the graph is as ever
    out = m.verify([0, 6], [-1, 0, 0, 1, 2, 2], [1, 2, 3, 4, 5, 6], x.cuda(), workspace(), temperatures=[1.0], uniforms=[0.3] * 6)
    m.status()
    path, token, _ = verify_exact([-1, 0, 0, 1, 2, 2], [1, 2, 3, 4, 5, 6], x, 1.0, [0.3] * 6)
    assert int(out[0][0]) == len(path) and int(out[2][0]) == token


def test_a_token_out_of_range_and_a_tree_of_too_many_nodes():
    V = 300
    m = TreeModel(n_q=2, n_kv=1, batch=4, max_seq=8, vocab=V, layers=1)
    x, work = torch.randn(260, V), workspace()
    x[0, 8] = 30.0
    for token in (-1, 300, 2 ** 31 - 1):
        out = m.verify([0, 3], [-1, 0, 0], [0, token, 8], x[:3].cuda(), work, temperatures=[1.0], uniforms=[0.5] * 3)
        with pytest.raises(M.MpkError, match=f"sequence 0 has token {token}"):
            m.status()
        m.graph.reset()
        assert out[1].tolist() == [0, 2, -1]   # never accepted; its sibling is
    out = m.verify([0, 257, 260], [-1] + [0] * 256 + [-1, 0, 0], [8] * 260, x.cuda(), work)
    with pytest.raises(M.MpkError, match="sequence 0 has a tree of 257 nodes"):
        m.status()
    m.graph.reset()
    assert out[0].tolist()[0] == 0 and int(out[2][0]) == -1 and (out[1][:257] == -1).all() and out[0].tolist()[1] >= 1


def test_no_rows_and_no_logprobs():
    m = TreeModel(n_q=2, n_kv=1, batch=4, max_seq=8, vocab=100, layers=1)
    b, n, t = m.ints([0, 0, 0]), m.ints([5, 5]), m.ints([5, 5])
    m.graph.tree_verify(2, 0, b.data_ptr(), 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, n.data_ptr(), 0, t.data_ptr(), 0, 0, torch.cuda.current_stream().cuda_stream)
    m.status()
    assert n.tolist() == [0, 0] and t.tolist() == [-1, -1]
    x = torch.randn(5, 100)
    for temp in (0.0, 1.0):
        outs = [m.verify([0, 5], [-1, 0, 0, 1, 1], [1, 2, 3, 4, 5], x.cuda(), workspace(), temperatures=[temp], uniforms=[0.4] * 5, logprobs=lp) for lp in (True, False)]
        m.status()
        assert all(torch.equal(a, b) for a, b in zip(outs[0][:3], outs[1][:3])) and (outs[1][3] == 77).all()


def test_rows_and_strides_far_apart():
    """Rows whose offsets pass 2^31 elements."""
    V, stride = 1000, 1 << 30
    m = TreeModel(n_q=2, n_kv=1, batch=4, max_seq=8, vocab=V, layers=1)
    x = torch.randn(5, V).to(torch.bfloat16)
    far = torch.empty(4 * stride + V, dtype=torch.bfloat16, device="cuda").as_strided((5, V), (stride, 1))
    far.copy_(x)
    tokens = [0] + [int(x[p].float().argmax()) for p in (0, 1, 2, 3)]
    out = m.verify([0, 5], [-1, 0, 1, 2, 3], tokens, far, workspace(), temperatures=[0.01], uniforms=[0.4] * 5)
    m.status()
    path, token, _ = verify_exact([-1, 0, 1, 2, 3], tokens, x, 0.01, [0.4] * 5)
    assert out[1].tolist() == path + [-1] * (5 - len(path)) and int(out[2][0]) == token and len(path) > 2


def test_the_same_call_gives_the_same_bits_two_graphs_at_once():
    """Calls of two graphs on two streams, many at a time, each with its workspace, against one after the other."""
    V, models = 50000, [TreeModel(n_q=2, n_kv=1, batch=8, max_seq=8, vocab=50000, layers=1) for _ in range(2)]
    gen, sets = torch.Generator().manual_seed(4), []
    for m in models:
        lens = [9, 30, 1, 12]
        begin, parents = _begin(lens), sum((tree(n, "random", i) for i, n in enumerate(lens)), [])
        x = (torch.randn(begin[-1], V, generator=gen) * 2).cuda()
        q = torch.softmax(x + torch.randn(begin[-1], V, generator=gen).cuda(), 1)
        tokens = _tokens(gen, x.cpu(), parents, begin, q.cpu(), True, None)
        sets.append((begin, parents, tokens, x, workspace(), q, True, [1.0] * 4, torch.rand(begin[-1], generator=gen)))
    want = [[t.clone() for t in m.verify(*s)] for m, s in zip(models, sets)]
    torch.cuda.synchronize()
    streams, got, keep = [torch.cuda.Stream() for _ in models], [[], []], []
    outs = [[[torch.empty_like(t).fill_(77) for t in w] for _ in range(20)] for w in want]
    torch.cuda.synchronize()
    for k in range(20):
        for j, (m, s) in enumerate(zip(models, sets)):
            with torch.cuda.stream(streams[j]):
                got[j].append(m.verify(*s, stream=streams[j].cuda_stream, out=outs[j][k]))
                keep.append(m.keep_alive)
    torch.cuda.synchronize()
    for m in models:
        m.status()
    for g, w in zip(got, want):
        for out in g:
            assert all(torch.equal(a, b) for a, b in zip(out, w))


def test_replays_between_other_calls_on_the_graph():
    """A captured call, replayed with new trees, logits and numbers, between calls of another number of sequences (other chunks) on the
    same graph, and after a reset."""
    V = 60000
    m = TreeModel(n_q=2, n_kv=1, batch=8, max_seq=8, vocab=V, layers=1)
    gen, work = torch.Generator().manual_seed(6), workspace()
    lens = [7, 12, 3]
    begin = _begin(lens)
    ints = [m.ints(x) for x in (begin, [-1] * 22, [0] * 22)]
    x, u, heat = torch.zeros(22, V, device="cuda"), torch.zeros(22, device="cuda"), torch.tensor([1.0, 0.0, 0.6], device="cuda")
    out = [m.ints([77] * 3), m.ints([77] * 22), m.ints([77] * 3), torch.full((22,), 77.0, device="cuda")]

    def call(stream):
        m.graph.tree_verify(3, 22, ints[0].data_ptr(), ints[1].data_ptr(), ints[2].data_ptr(), x.data_ptr(), M.ROWS_F32, V, 0, 0, 0, heat.data_ptr(), u.data_ptr(),
                            *[t.data_ptr() for t in out], work.data_ptr(), stream)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(torch.cuda.current_stream().cuda_stream)
    for n in range(6):
        parents = sum((tree(k, "random", 10 * n + i) for i, k in enumerate(lens)), [])
        logits, uniforms = torch.randn(22, V, generator=gen) * 2, torch.rand(22, generator=gen)
        logits[torch.arange(22), torch.randint(V, (22,), generator=gen)] += 14
        tokens = _tokens(gen, logits, parents, begin, None, False, None)
        ints[1].copy_(m.ints(parents)), ints[2].copy_(m.ints(tokens)), x.copy_(logits), u.copy_(uniforms)
        for t in out:
            t.fill_(77)
        graph.replay()
        m.status()
        _check(m, begin, parents, tokens, logits, out, heat.tolist(), uniforms)
        sub = slice(begin[n % 3], begin[n % 3 + 1])   # one of the sequences alone, its row in chunks of its own
        alone = m.verify([0, lens[n % 3]], parents[sub], tokens[sub], x[sub].clone(), work, temperatures=[1.0], uniforms=uniforms[sub])
        m.status()
        _check(m, [0, lens[n % 3]], parents[sub], tokens[sub], logits[sub], alone, [1.0], uniforms[sub])
        if n == 3:
            m.graph.reset()


@pytest.mark.parametrize("draft", [None, "once"])
def test_beside_work_that_fills_the_gpu(draft):
    """Products on another stream hold compute units, so that a call's workgroups do not all run at once: the same results, in time."""
    V, lens = 120001, [9, 1, 14, 5, 0, 3, 7, 2]
    m = TreeModel(n_q=2, n_kv=1, batch=8, max_seq=8, vocab=V, layers=1)
    gen = torch.Generator().manual_seed(8)
    begin, parents = _begin(lens), sum((tree(n, "random", i) for i, n in enumerate(lens)), [])
    x = torch.randn(begin[-1], V, generator=gen) * 2
    x[torch.arange(begin[-1]), torch.randint(V, (begin[-1],), generator=gen)] += 12
    q = torch.softmax(x + torch.randn(begin[-1], V, generator=gen), 1) if draft else None
    tokens, uniforms, temps = _tokens(gen, x, parents, begin, q, True, None), torch.rand(begin[-1], generator=gen), [1.0, 0.0, 0.8, 1.2] * 2
    logits, probs, work = x.cuda(), q.cuda() if draft else None, workspace()
    a, other = torch.randn(6000, 6000, device="cuda", dtype=torch.bfloat16), torch.cuda.Stream()
    outs, keep = [], []
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(other):
            for _ in range(4):
                b = a @ a
        for _ in range(3):
            outs.append(m.verify(begin, parents, tokens, logits, work, probs, draft == "once", temps, uniforms))
            keep.append(m.keep_alive)
    torch.cuda.synchronize()
    m.status()
    for out in outs:
        assert all(torch.equal(p.view(torch.int32), r.view(torch.int32)) for p, r in zip(out, outs[0]))
    _check(m, begin, parents, tokens, x, outs[0], temps, uniforms, q, draft == "once")


BELOW_ONE = 1 - 2 ** -24


def _places(vocab, n):
    """n tokens that lie in many chunks of a row: its first and last among them."""
    return [0] if n == 1 else [i * (vocab - 1) // (n - 1) for i in range(n)]


def _star(m, x, children, uniforms, temperature=1.0):
    """Children of a root, against the definition.  Their own rows are flat: with V equal weights the first v with (v + 1) / V > u is floor(u V),
    in whole numbers here (a sum of rounded shares may lie on either side where u V is whole)."""
    V, nodes = x.shape[0], 1 + len(children)
    logits = torch.zeros(nodes, V)
    logits[0] = x
    parents, tokens = [-1] + [0] * len(children), [0] + children
    out = m.verify([0, nodes], parents, tokens, logits.cuda(), workspace(), temperatures=[temperature], uniforms=uniforms)
    m.status()
    walk, token, logs = verify_exact(parents, tokens, logits, temperature, uniforms)
    if len(walk) == 2:
        token = int(Fraction(float(torch.tensor(uniforms[0]))) * V)
    rest = nodes - len(walk)
    assert [int(out[0][0]), out[1].tolist(), int(out[2][0])] == [len(walk), walk + [-1] * rest, token]
    want = torch.tensor(logs + [0.0] * rest, dtype=torch.float64)
    assert ((out[3].cpu().double() - want).abs() <= F32_HALF * want.abs() + 2e-9).all()   # as in _check
    return out


@pytest.mark.parametrize("vocab", [0, 700, 5000, 150001])   # 0: the tokens alone
@pytest.mark.parametrize("gaps,u", [
    # a child that holds all but some 1e-7 of what is left is refused by the largest number below one; the last one is left alone
    ([16.1], [BELOW_ONE, BELOW_ONE]), ([16.125, 16.125], [BELOW_ONE, BELOW_ONE, 0.5]), ([16.125, 16.125], [BELOW_ONE] * 3),
    ([16.5] * 11, [BELOW_ONE] * 11 + [0.5]), ([16.5] * 11, [BELOW_ONE] * 12),
    # large shares, refused by numbers of the ordinary size; then two alike
    ([2.0, 3.0, 1.5, 4.0], [0.95, 0.97, 0.9, 0.99, BELOW_ONE]), ([16.5, 16.5, 0.0], [BELOW_ONE, BELOW_ONE, 0.75, BELOW_ONE])])
def test_children_that_hold_all_there_is(gaps, u, vocab):
    """Every token that is not ruled out is a child: the walk goes on at one of them, whatever the numbers."""
    heights = [0.0]
    for g in gaps:
        heights.append(heights[-1] - g)
    V = vocab or len(heights)
    x, at = torch.full((V,), -math.inf), _places(V, len(heights))
    x[at] = torch.tensor(heights)
    out = _star(TreeModel(n_q=2, n_kv=1, batch=4, max_seq=8, vocab=V, layers=1), x, at, [0.5] + u)
    assert int(out[0][0]) == 2 and int(out[2][0]) >= 0


@pytest.mark.parametrize("root", [0.0, 0.3, 0.8, BELOW_ONE])
@pytest.mark.parametrize("vocab", [40, 3000, 70001])
@pytest.mark.parametrize("children,gap", [(1, 16.5), (2, 16.5), (7, 16.25), (3, 7.0), (1, 7.0)])
def test_tokens_behind_children_that_hold_nearly_all(children, gap, vocab, root):
    """Refused children leave tokens of much less probability than the row began with; one is drawn, in chunks of the children and others."""
    gen = torch.Generator().manual_seed(children + vocab)
    low = -gap * children
    x, at = low + torch.randn(vocab, generator=gen) - math.log(vocab), _places(vocab, children)
    x[at] = -gap * torch.arange(children, dtype=torch.float32)
    out = _star(TreeModel(n_q=2, n_kv=1, batch=4, max_seq=8, vocab=vocab, layers=1), x, at, [root] + [BELOW_ONE] * children)
    assert int(out[0][0]) == 1 and int(out[2][0]) not in at


@pytest.mark.parametrize("last", [0.5, BELOW_ONE])
@pytest.mark.parametrize("order", range(4))
def test_children_in_many_groups_hold_all_there_is(order, last):
    """As above with 255 children: unlikely ones, twins and out of turn, around a few that hold nearly all."""
    V, rng = 9000, random.Random(order)
    heavy = [rng.randrange(V) for _ in range(5)]
    light = [t for t in rng.sample(range(V), 260) if t not in heavy][:100]
    children = light + [rng.choice(light) for _ in range(255 - 5 - 20 - len(light))]
    for h in heavy:   # in ascending order of their places, twins of them behind them
        children.insert(rng.randrange(40) + 45 * heavy.index(h), h)
    behind = max(children.index(h) for h in heavy)
    for _ in range(20):
        children.insert(rng.randint(behind + 1, len(children)), rng.choice(heavy[:4]))
    x = torch.full((V,), -math.inf)
    x[light] = -120.0 - torch.rand(len(light), generator=torch.Generator().manual_seed(order))
    turn = sorted(heavy, key=children.index)
    x[turn] = -16.5 * torch.arange(5, dtype=torch.float32)
    u = [0.5] + [BELOW_ONE if c in heavy else 0.6 for c in children]
    u[1 + children.index(turn[-1])] = last
    out = _star(TreeModel(n_q=2, n_kv=1, batch=4, max_seq=8, vocab=V, layers=1), x, children, u)
    assert out[1].tolist()[1] == 1 + children.index(turn[-1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("temperatures", [[1.0], [0.5, 1.0, 0.0, 2.0]])
def test_walks_through_nodes_whose_children_hold_nearly_all(temperatures, dtype):
    """Several sequences, late workgroups: at each node a few tokens in steps of some 16 temperatures, the likeliest first among the children,
    numbers that refuse most of them."""
    V, lens, gen = 30011, [12, 1, 40, 9, 25], torch.Generator().manual_seed(2)
    m = TreeModel(n_q=2, n_kv=1, batch=8, max_seq=8, vocab=V, layers=1, debug_flags=M.DEBUG_JITTER)
    begin, parents = _begin(lens), sum((tree(n, "random", 50 + i) for i, n in enumerate(lens)), [])
    x = torch.full((begin[-1], V), -math.inf)
    tokens, uniforms, temps = [0] * begin[-1], [0.37] * begin[-1], [temperatures[i % len(temperatures)] for i in range(len(lens))]
    for i in range(len(lens)):
        kids = {}
        for t in range(begin[i], begin[i + 1]):
            row = torch.randperm(V, generator=gen)
            step = 16.5 * (temps[i] or 1.0)
            x[t, row[:6]] = -step * torch.arange(6, dtype=torch.float32)
            x[t, row[6:400]] = -6 * step + torch.randn(394, generator=gen) - 8.0
            p = parents[t]
            if p >= 0:
                j = kids[p] = kids.get(p, -1) + 1
                order = x[begin[i] + p].sort(descending=True).indices
                tokens[t] = int(order[min(j, 5)])
                uniforms[t] = BELOW_ONE if (t + j) % 3 else 0.61
    logits = x.to(dtype)
    for _ in range(3):
        out = m.verify(begin, parents, tokens, logits.cuda(), workspace(), temperatures=temps, uniforms=uniforms)
        m.status()
        _check(m, begin, parents, tokens, logits, out, temps, torch.tensor(uniforms), None)


def test_equal_shares_are_exact():
    """Of eight equal tokens four are refused: u = 1/4 refuses the fifth (u q < r is strict), the number in front of it accepts."""
    m = TreeModel(n_q=2, n_kv=1, batch=4, max_seq=8, vocab=8, layers=1)
    for u, length in ((0.25, 1), (0.25 - 2 ** -26, 2)):
        out = m.verify([0, 6], [-1, 0, 0, 0, 0, 0], [0, 7, 1, 4, 2, 3], torch.full((6, 8), 3.25).cuda(), workspace(), temperatures=[1.3],
                       uniforms=[0.0] + [BELOW_ONE] * 4 + [u])
        m.status()
        assert int(out[0][0]) == length
        assert length == 2 or int(out[2][0]) == 0


@pytest.mark.parametrize("draft", [None, "drawn"])
def test_verify_rows_of_many_steps_a_workgroup(draft):
    """Sixteen rows of 1.2 million logits, 13 steps of a workgroup each: chunks that take longer than others wait by default."""
    lens = [2, 1, 1, 3, 1, 1, 2, 1, 1, 1, 2, 1, 1, 1, 1, 1]
    _case(12, 1200000, lens, ["chain"] * 16, torch.bfloat16, draft, [1.0, 0.8, 0.0], std=3.0)


@pytest.mark.parametrize("root", [0.0, 2 ** -24, 0.4, BELOW_ONE])
@pytest.mark.parametrize("low", [-40.0, -90.0, -math.inf])
@pytest.mark.parametrize("heavy", [[1055, 3388], [3388, 1055], [0, 2047, 4999], [2100, 2101, 2102, 4100], [4999, 0, 4998]])
def test_a_chunk_that_its_refused_tokens_leave_hardly_anything_of(heavy, low, root):
    """All but the last of the likely tokens are refused, by ordinary numbers: u = 0 draws the first token that has any probability, of a chunk
    whose sum does not show it too."""
    V, gen = 5000, torch.Generator().manual_seed(len(heavy))
    x = low + torch.randn(V, generator=gen) if low > -math.inf else torch.full((V,), low)
    x[heavy] = 0.7 + 0.01 * torch.arange(len(heavy)).float()
    out = _star(TreeModel(n_q=2, n_kv=1, batch=4, max_seq=8, vocab=V, layers=1), x, heavy[:-1], [root] + [0.75] * (len(heavy) - 1))
    assert int(out[0][0]) == 1
    if root == 0.0:
        first = 1 if 0 in heavy[:-1] else 0
        assert int(out[2][0]) == (first if low > -math.inf else heavy[-1])
