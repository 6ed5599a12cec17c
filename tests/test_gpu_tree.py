"""mpk_tree_append, mpk_tree_attend and mpk_tree_keep on the GPU against 64-bit results, and the four calls together."""
import random
from types import SimpleNamespace

import pytest
import torch

import paper_2512_22219_amd as M
from tests.rows_util import append_exact
from tests.tree_util import BF16_HALF, F32_HALF, TreeModel, chains, tree, tree_attend_exact, workspace

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.contiguous().view(torch.int16)


def _begin(lens, first=0):
    out = [first]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _forest(lens, kinds, behind=0, first=0, seed=0):
    """Parents of all rows of a call, and of each sequence."""
    each = [tree(n, k, seed + i, roots=2 if k == "roots" else 1) for i, (n, k) in enumerate(zip(lens, kinds))]
    return [99] * first + sum(each, []) + [-99] * behind, each


APPEND = [
    dict(n_q=4, n_kv=2, d=64, lens=[1], pos=[0], slots=None, kinds=["chain"]),
    dict(n_q=8, n_kv=8, d=128, lens=[3, 0, 2], pos=[7, 191, 190], slots=[2, 0, 1], kinds=["star", "chain", "roots"], qk_norm=True),
    dict(n_q=16, n_kv=2, d=64, lens=[33, 64, 5, 90], pos=[0, 128, 60, 101], slots=[3, 2, 1, 0], kinds=["two", "random", "star", "chain"], theta=1e6,
         first=2, behind=3),
    dict(n_q=16, n_kv=2, d=128, lens=[0, 17], pos=[5, 11], slots=None, kinds=["chain", "random"], qk_norm=True, page=8, pages=101, behind=5),
    dict(n_q=4, n_kv=1, d=128, lens=[100, 92, 65, 1], pos=[92, 0, 100, 64], slots=[1, 0, 3, 2], kinds=["random"] * 4, page=64, pages=13, first=1),
    dict(n_q=32, n_kv=8, d=128, lens=[256, 200, 129], pos=[3700, 0, 17], slots=None, kinds=["chain", "random", "two"], max_seq=4096, batch=3,
         layers=2, qk_norm=True, theta=5e5),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad", [0, 24])
@pytest.mark.parametrize("case", APPEND)
def test_append(case, pad, dtype):
    c = dict(case)
    lens, pos, slots, kinds, first, behind = c.pop("lens"), c.pop("pos"), c.pop("slots"), c.pop("kinds"), c.pop("first", 0), c.pop("behind", 0)
    m = TreeModel(**c)
    begin = _begin(lens, first)
    parents, each = _forest(lens, kinds, behind, first)
    rows, heads = begin[-1] + behind, m.n_q + 2 * m.n_kv
    x = m.normal(rows, heads * m.d + pad, dtype=torch.float32).to(dtype)
    q_out = m.normal(rows, m.n_q * m.d + pad)
    q0, k0, v0 = q_out.clone(), m.k.clone(), m.v.clone()
    m.tree_append(1, begin, slots, pos, parents, x, q_out)
    m.status()
    k1, v1, q1 = k0.clone(), v0.clone(), q0.clone()
    for i, (n, p) in enumerate(zip(lens, pos)):
        if not n:
            continue
        r = slice(begin[i], begin[i + 1])
        at = torch.arange(p, p + n, device=m.dev)
        turn = torch.tensor([p + len(a) - 1 for a in chains(each[i])], device=m.dev)
        q, k, v, q_size, k_size = append_exact(m, 1, turn, x[r, : heads * m.d])
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


def test_a_chain_is_a_prompt():
    """Chains through the calls on trees and the same rows through the calls on rows: the same bits appended, and outputs that are as
    near to the same results in 64 bits (keys may be added up in another order)."""
    kw = dict(n_q=8, n_kv=2, d=128, qk_norm=True, max_seq=704, batch=3, layers=1, seed=3)
    a, b = TreeModel(**kw), TreeModel(**kw)
    lens, pos = [37, 1, 256], [400, 77, 191]
    begin, (parents, _) = _begin(lens), _forest(lens, ["chain"] * 3)
    x = a.normal(begin[-1], 12 * 128)
    q, o, work = torch.empty(2, begin[-1], 1024, dtype=torch.bfloat16, device=a.dev), torch.empty(2, begin[-1], 1024, dtype=torch.bfloat16, device=a.dev), workspace()
    a.tree_append(0, begin, None, pos, parents, x, q[0])
    b.append(0, begin, None, pos, x, q[1])
    a.tree_attend(0, begin, None, pos, parents, q[0], o[0], work)
    a.status()
    b.attend(0, begin, None, pos, q[1], o[1], work)
    b.status()
    assert torch.equal(_bits(q[0]), _bits(q[1])) and torch.equal(_bits(a.k), _bits(b.k)) and torch.equal(_bits(a.v), _bits(b.v))
    each = [tree(n, "chain") for n in lens]
    for m, out in ((a, o[0]), (b, o[1])):
        _check_attend(m, 0, lens, pos, None, begin, each, q[0], out)


def test_append_in_place():
    m = TreeModel(n_q=8, n_kv=2, d=64, qk_norm=True, max_seq=400, batch=3, page=16, pages=80)
    lens, pos = [250, 0, 140], [100, 3, 201]
    begin, (parents, _) = _begin(lens), _forest(lens, ["random"] * 3)
    x = m.normal(begin[-1], 12 * 64)
    q = torch.empty(begin[-1], 512, dtype=torch.bfloat16, device=m.dev)
    m.tree_append(0, begin, None, pos, parents, x, q)
    k0, v0, y = m.k.clone(), m.v.clone(), x.clone()
    m.tree_append(0, begin, None, pos, parents, y, y)
    m.status()
    assert torch.equal(_bits(y[:, :512]), _bits(q)) and torch.equal(_bits(y[:, 512:]), _bits(x[:, 512:]))
    assert torch.equal(_bits(k0), _bits(m.k)) and torch.equal(_bits(v0), _bits(m.v))


ATTEND = [
    dict(n_q=4, n_kv=2, d=64, lens=[1], pos=[0], slots=None, kinds=["chain"]),                       # one node, nothing cached
    dict(n_q=8, n_kv=8, d=128, lens=[1, 1, 1], pos=[0, 63, 191], slots=[1, 2, 0], kinds=["chain"] * 3),
    dict(n_q=8, n_kv=1, d=128, lens=[2, 0, 3], pos=[64, 3, 126], slots=None, kinds=["roots", "chain", "roots"]),
    dict(n_q=16, n_kv=2, d=64, lens=[5, 7], pos=[187, 62], slots=[3, 1], kinds=["star", "two"], first=2, behind=3),
    dict(n_q=8, n_kv=2, d=128, lens=[64], pos=[0], slots=None, kinds=["random"]),
    dict(n_q=4, n_kv=4, d=64, lens=[65, 1, 130], pos=[0, 100, 61], slots=[2, 0, 3], kinds=["two", "chain", "star"], behind=1),
    dict(n_q=16, n_kv=2, d=128, lens=[129, 17, 0, 1], pos=[40, 0, 0, 9], slots=None, kinds=["random"] * 4, page=8, pages=97),
    dict(n_q=8, n_kv=8, d=64, lens=[192, 33], pos=[0, 159], slots=[1, 0], kinds=["roots", "random"], page=16, pages=48, first=1),
    dict(n_q=2, n_kv=1, d=128, lens=[256], pos=[448], slots=None, kinds=["random"], max_seq=704, batch=1),
    dict(n_q=4, n_kv=1, d=64, lens=[256, 255], pos=[1500, 1001], slots=[1, 0], kinds=["chain", "two"], max_seq=1808, batch=2),
    dict(n_q=32, n_kv=8, d=128, lens=[1, 2], pos=[5000, 17], slots=None, kinds=["chain", "roots"], max_seq=5056, batch=2, page=64, pages=160, layers=1),
    dict(n_q=8, n_kv=1, d=64, lens=[4], pos=[20003], slots=None, kinds=["star"], max_seq=20008, batch=1, layers=1),
    dict(n_q=32, n_kv=4, d=128, lens=[1, 40, 200, 8, 1, 256, 9, 1], pos=[1000, 0, 300, 500, 0, 0, 31, 1022], slots=[7, 6, 5, 4, 3, 2, 1, 0],
         kinds=["chain", "random", "random", "star", "chain", "random", "two", "chain"], max_seq=1024, batch=8, layers=1),
    dict(n_q=8, n_kv=1, d=128, lens=[256], pos=[3744], slots=[0], kinds=["random"], max_seq=4000, batch=1, layers=1),
    dict(n_q=8, n_kv=4, d=128, lens=[63, 64, 65, 31] * 4, pos=[1, 2, 63, 64, 127, 128, 129, 190, 500, 511, 513, 575, 576, 700, 701, 1800], slots=None,
         kinds=["random"] * 16, max_seq=1864, batch=16, layers=1),
]


def _attend_case(case, pad=0, seed=0):
    c = dict(case)
    lens, pos, slots, kinds, first, behind = c.pop("lens"), c.pop("pos"), c.pop("slots"), c.pop("kinds"), c.pop("first", 0), c.pop("behind", 0)
    m = TreeModel(seed=seed, **c)
    begin = _begin(lens, first)
    parents, each = _forest(lens, kinds, behind, first, seed)
    q = m.normal(begin[-1] + behind, m.n_q * m.d + pad)
    return m, lens, pos, slots, begin, parents, each, q


def _check_attend(m, layer, lens, pos, slots, begin, each, q, out, before=None, clean=None):
    """clean: caches to take the results from, where the model's hold what no node sees."""
    k, v = clean or (m.k, m.v)
    for i, (n, p) in enumerate(zip(lens, pos)):
        if not n:
            continue
        r, slot = slice(begin[i], begin[i + 1]), slots[i] if slots else i
        width = m.n_q * m.d
        want, bound = tree_attend_exact(q[r, :width].view(n, m.n_q, m.d), m.cached(k, layer, slot, p + n), m.cached(v, layer, slot, p + n), p, each[i])
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
    m, lens, pos, slots, begin, parents, each, q = _attend_case(case, pad)
    out = m.normal(q.shape[0], m.n_q * m.d + pad)
    before = out.clone()
    layer = m.layers - 1
    m.tree_attend(layer, begin, slots, pos, parents, q, out, workspace())
    m.status()
    _check_attend(m, layer, lens, pos, slots, begin, each, q, out, before)


def _random_case(seed):
    rng = random.Random(seed)
    n_kv = rng.choice([1, 2, 4, 8])
    batch = rng.choice([1, 2, 3, 7, 16])
    page = rng.choice([0, 0, 8, 32, 64])
    max_seq = 64 * rng.randint(5, 40)
    lens = [rng.choice([0, 1, rng.randint(1, 9), rng.randint(1, 64), rng.randint(1, 256)]) for _ in range(batch)]
    pos = [rng.randint(0, max_seq - max(n, 1)) for n in lens]
    slots = rng.choice([None, rng.sample(range(batch), batch)])
    c = dict(n_q=n_kv * rng.choice([1, 2, 4, 8]), n_kv=n_kv, d=rng.choice([64, 128]), batch=batch, max_seq=max_seq, layers=1, lens=lens, pos=pos,
             slots=slots, kinds=[rng.choice(["chain", "star", "two", "random", "random", "roots"]) for _ in lens], first=rng.choice([0, 3]),
             behind=rng.choice([0, 2]))
    if page:
        c.update(page=page, pages=batch * (max_seq // page) + 5)
    return c


@pytest.mark.parametrize("seed", range(40))
def test_random_trees(seed):
    case = _random_case(seed)
    m, lens, pos, slots, begin, parents, each, q = _attend_case(case, seed=seed)
    x = m.normal(q.shape[0], (m.n_q + 2 * m.n_kv) * m.d)
    out = m.normal(q.shape[0], m.n_q * m.d)
    m.tree_append(0, begin, slots, pos, parents, x, q)
    before = out.clone()
    m.tree_attend(0, begin, slots, pos, parents, q, out, workspace())
    m.status()
    _check_attend(m, 0, lens, pos, slots, begin, each, q, out, before)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("case", [ATTEND[i] for i in (1, 3, 4, 5, 6, 9, 12, 14)])
def test_what_a_node_does_not_see_never_reaches_it(case, bad):
    """Everything behind the trees, and the rows of one node (and its descendants) of each, hold what is not finite: the other nodes
    are as if it were not there."""
    m, lens, pos, slots, begin, parents, each, q = _attend_case(case)
    layer, clean, work = m.layers - 1, (m.k.clone(), m.v.clone()), workspace()
    out = m.normal(q.shape[0], m.n_q * m.d)
    spoilt = []
    for i, (n, p) in enumerate(zip(lens, pos)):
        slot = slots[i] if slots else i
        hit = n // 2
        spoilt.append([hit in c for c in chains(each[i])] if n else [])
        rows = ([p + hit] if n else []) + list(range(p + n, m.max_seq))
        rows = torch.tensor(rows, dtype=torch.long, device=m.dev)
        for cache in (m.k, m.v):
            if m.page:
                cache[layer][m.table[slot].long()[rows // m.page], :, rows % m.page] = bad
            else:
                cache[layer, slot][:, rows] = bad
    assert not m.page or len(set(m.table.flatten().tolist())) == m.table.numel()   # (no page is two sequences')
    m.tree_attend(layer, begin, slots, pos, parents, q, out, work)
    m.status()
    for i, (n, p) in enumerate(zip(lens, pos)):
        fine = [t for t in range(n) if not spoilt[i][t]]
        if not fine:
            continue
        slot = slots[i] if slots else i
        want, bound = tree_attend_exact(q[begin[i]:begin[i + 1]].view(n, m.n_q, m.d), m.cached(clean[0], layer, slot, p + n),
                                        m.cached(clean[1], layer, slot, p + n), p, each[i])
        got = out[begin[i]:begin[i + 1]].view(n, m.n_q, m.d).double()
        assert ((got - want).abs() / bound)[fine].max() <= 1


def test_a_value_that_is_not_finite_reaches_the_nodes_that_see_it():
    m = TreeModel(n_q=4, n_kv=1, d=128, max_seq=256, batch=1, layers=1)
    parents = tree(90, "random", 4)
    q, out = m.normal(90, 512), torch.empty(90, 512, dtype=torch.bfloat16, device="cuda")
    m.v[0, 0, 0, 100 + 30, 5] = float("inf")
    m.v[0, 0, 0, 100 + 41, 6] = float("nan")
    m.tree_attend(0, [0, 90], None, [100], parents, q, out, workspace())
    m.status()
    out = out.view(90, 4, 128)
    for t, chain in enumerate(chains(parents)):
        assert (out[t, :, 5] == float("inf")).all() == (30 in chain) and torch.isnan(out[t, :, 6]).all() == (41 in chain)
        rest = [c for c in range(128) if not (c == 5 and 30 in chain) and not (c == 6 and 41 in chain)]
        assert torch.isfinite(out[t][:, rest]).all()


@pytest.mark.parametrize("page", [0, 4096])
def test_a_cache_whose_offsets_pass_32_bits(page):
    """The last slot of a cache of more than 2^32 elements, one layer."""
    batch, n_kv, d, max_seq = 16, 4, 128, 589824
    assert batch * n_kv * d * max_seq > 1 << 32
    kw = dict(page=page, pages=batch * max_seq // page) if page else {}
    m = TreeModel(n_q=8, n_kv=n_kv, d=d, layers=1, batch=batch, max_seq=max_seq, fill=0.0, **kw)
    n, p = 70, max_seq - 70
    parents = tree(n, "random", 2)
    x, q, out = m.normal(n, (8 + 2 * n_kv) * d), m.normal(n, 8 * d), m.normal(n, 8 * d)
    if page:
        m.table.copy_(torch.arange(m.table.numel(), dtype=torch.int32, device=m.dev).view(m.table.shape))
    m.tree_append(0, [0, n], [15], [p], parents, x, q)
    m.tree_attend(0, [0, n], [15], [p], parents, q, out, workspace())
    m.status()
    k, v = (m.cached(c, 0, 15, max_seq)[:, p:].double() for c in (m.k, m.v))
    _, rk, rv, _, size = append_exact(m, 0, torch.tensor([p + len(c) - 1 for c in chains(parents)], device=m.dev), x)
    assert ((k.transpose(0, 1) - rk).abs() <= BF16_HALF * rk.abs() + 48 * F32_HALF * size).all() and torch.equal(v.transpose(0, 1), rv)
    # cached rows of zeros: score 0, value 0
    qd, seen = q.view(n, n_kv, 2, d).double().permute(1, 0, 2, 3), torch.zeros(n, n, dtype=torch.bool)
    for t, c in enumerate(chains(parents)):
        seen[t, c] = True
    s = (qd @ k[:, None].transpose(2, 3).contiguous() / d ** 0.5).exp() * seen.to(m.dev)[None, :, None]
    want = (s @ v[:, None]) / (s.sum(-1, keepdim=True) + p)
    size = (s @ v[:, None].abs()) / (s.sum(-1, keepdim=True) + p)
    got = out.view(n, n_kv, 2, d).double().permute(1, 0, 2, 3)
    # the weights of 2^19 equal rows add up to 2^-12 relative at the worst of a lane's 32-bit sum
    assert ((got - want).abs() <= BF16_HALF * want.abs() + (BF16_HALF + 2 ** -12) * size).all()
    m.keep([0, n], [15], [p], [3], [0, 5, 69] + [-1] * 67)
    m.status()
    for cache, old in ((m.k, k), (m.v, v)):
        new = m.cached(cache, 0, 15, max_seq)[:, p:].double()
        assert torch.equal(new[:, 1], old[:, 5]) and torch.equal(new[:, 2], old[:, 69]) and torch.equal(new[:, 3:], old[:, 3:])


def _kept(m, lens, pos, slots, begin, path, lengths, k0, v0):
    """The caches that keep should leave."""
    k1, v1 = k0.clone(), v0.clone()
    for i, (n, p) in enumerate(zip(lens, pos)):
        slot = slots[i] if slots else i
        for k in range(lengths[i]):
            t = path[begin[i] + k]
            for new, old in ((k1, k0), (v1, v0)):
                if m.page:
                    tab = m.table[slot].tolist()
                    new[:, tab[(p + k) // m.page], :, (p + k) % m.page] = old[:, tab[(p + t) // m.page], :, (p + t) % m.page]
                else:
                    new[:, slot, :, p + k] = old[:, slot, :, p + t]
    return k1, v1


@pytest.mark.parametrize("kw", [dict(n_q=4, n_kv=2, d=64), dict(n_q=8, n_kv=8, d=128, layers=5), dict(n_q=4, n_kv=1, d=128, page=8, pages=400),
                                dict(n_q=16, n_kv=2, d=64, page=64, pages=60, layers=3), dict(n_q=3, n_kv=3, d=64, layers=1)])
@pytest.mark.parametrize("seed", range(6))
def test_keep(kw, seed):
    rng = random.Random(seed)
    m = TreeModel(batch=5, max_seq=512, seed=seed, **kw)
    lens = [rng.choice([0, 1, 2, 17, 64, 65, 200, 256]) for _ in range(5)]
    pos = [rng.choice([0, 1, 255, rng.randint(0, 512 - max(n, 1)), 512 - max(n, 1)]) for n in lens]
    pos = [min(p, 512 - n) for p, n in zip(pos, lens)]
    pos = [min(p, 511) for p in pos]
    slots = rng.choice([None, rng.sample(range(5), 5)])
    begin = _begin(lens, 2)
    lengths = [rng.choice([0, 1, n, rng.randint(1, n), min(n, 3)]) if n else 0 for n in lens]
    path = [-7, -7]
    for n, k in zip(lens, lengths):
        path += (sorted(rng.sample(range(n), k)) if rng.random() < 0.8 else list(range(k))) + [-1] * (n - k)
    path += [-7] * 3
    k0, v0, ends = m.k.clone(), m.v.clone(), torch.full((6,), 55, dtype=torch.int32, device="cuda")
    m.keep(begin, slots, pos, lengths, path, ends)
    m.status()
    k1, v1 = _kept(m, lens, pos, slots, begin, path, lengths, k0, v0)
    assert torch.equal(_bits(k1), _bits(m.k)) and torch.equal(_bits(v1), _bits(m.v))
    assert ends.tolist() == [p + n for p, n in zip(pos, lengths)] + [55]


# what the device finds: begin, slots, positions, sequences left out, what the status says
WRONG = [
    (dict(begin=[0, 3, 2, 6]), {0, 1, 2}, "row_begin.*sequence 1"),
    (dict(begin=[-1, 3, 4, 6]), {0, 1, 2}, "row_begin.*sequence 0"),
    (dict(begin=[0, 3, 4, 7]), {0, 1, 2}, "row_begin.*sequence 2"),
    (dict(slots=[0, 4, 2]), {1}, "sequence 1 has slot 4"),
    (dict(slots=[2, 1, 2]), {2}, "sequence 2 has slot 2"),
    (dict(positions=[-1, 0, 0]), {0}, "sequence 0 has position -1"),
    (dict(positions=[0, 0, 191]), {2}, "sequence 2 has position 192"),
    (dict(parents=[0, 0, 0, -1, -1, 0]), {0}, "sequence 0: node 0"),
    (dict(parents=[-1, 0, 2, -1, -1, 0]), {0}, "sequence 0: node 2"),
    (dict(parents=[-1, 0, 1, -1, -1, 5]), {2}, "sequence 2: node 1"),
    (dict(parents=[-1, 0, 1, -2, -1, 0]), {1}, "sequence 1: node 0"),
]


@pytest.mark.parametrize("change,left,says", WRONG)
def test_wrong_sequences_are_reported_and_left_out(change, left, says):
    m = TreeModel(n_q=4, n_kv=2, d=64, batch=4)
    args = dict(dict(begin=[0, 3, 4, 6], slots=[0, 1, 2], positions=[5, 6, 7], parents=[-1, 0, 0, -1, -1, 0]), **change)
    begin, slots, pos, parents = args.values()
    x, q, o = m.normal(6, 8 * 64), m.normal(6, 256), m.normal(6, 256)
    q0, o0, k0 = q.clone(), o.clone(), m.k.clone()

    def check(call, out, out0):
        call()
        with pytest.raises(M.MpkError, match=says) as e:
            m.status()
        assert e.value.status == M.MPK_ERR_DEVICE
        m.graph.reset()
        m.status()
        for i in range(3):
            r = slice(max(0, begin[i]), begin[i + 1])
            if out is not None and i in left:
                assert torch.equal(_bits(out[r]), _bits(out0[r]))
            elif out is not None:
                assert not torch.equal(_bits(out[r]), _bits(out0[r])) or begin[i] == begin[i + 1]

    check(lambda: m.tree_append(1, begin, slots, pos, parents, x, q), q, q0)
    for i in range(3):
        if i not in left:
            k0[1, slots[i]] = m.k[1, slots[i]]
    assert torch.equal(_bits(k0), _bits(m.k))
    wrong_tree = "parents" in change   # (the outputs are undefined then)
    check(lambda: m.tree_attend(1, begin, slots, pos, parents, q, o, workspace()), None if wrong_tree else o, o0)
    if not wrong_tree:
        k0, ends = m.k.clone(), torch.full((3,), -5, dtype=torch.int32, device="cuda")
        check(lambda: m.keep(begin, slots, pos, [2, 1, 1], [0, 2, -1, 0, 1, -1], ends), None, None)
        assert ends.tolist() == [p if i in left else p + n for i, (p, n) in enumerate(zip(pos, [2, 1, 1]))]
        for i in range(3):
            if i not in left:
                k0[:, slots[i]] = m.k[:, slots[i]]
        assert torch.equal(_bits(k0), _bits(m.k))


def test_trees_of_too_many_nodes_are_reported_and_left_out():
    m = TreeModel(n_q=4, n_kv=2, d=64, batch=2, max_seq=400)
    begin, parents = [0, 257, 260], [-1] + [0] * 256 + [-1, 0, 0]
    x, q, o = m.normal(260, 8 * 64), m.normal(260, 256), m.normal(260, 256)
    q0, o0, k0, ends = q.clone(), o.clone(), m.k.clone(), torch.zeros(2, dtype=torch.int32, device="cuda")
    for call, out, out0 in ((lambda: m.tree_append(0, begin, None, [3, 4], parents, x, q), q, q0),
                            (lambda: m.tree_attend(0, begin, None, [3, 4], parents, q, o, workspace()), o, o0),
                            (lambda: m.keep(begin, None, [3, 4], [2, 2], [0, 9] + [-1] * 255 + [0, 2, -1], ends), None, None)):
        call()
        with pytest.raises(M.MpkError, match="sequence 0 has a tree of 257 nodes"):
            m.status()
        m.graph.reset()
        if out is not None:
            assert torch.equal(_bits(out[:257]), _bits(out0[:257])) and not torch.equal(_bits(out[257:]), _bits(out0[257:]))
    assert torch.equal(_bits(m.k[:, 0]), _bits(k0[:, 0])) and ends.tolist() == [3, 6]


@pytest.mark.parametrize("lengths,path,says", [
    ([4, 1], [0, 1, 2, 0, -1], "sequence 0"), ([-1, 1], [0, 1, 2, 0, -1], "sequence 0"), ([2, 1], [1, 1, -1, 0, -1], "sequence 0: place 1"),
    ([2, 1], [1, 0, -1, 0, -1], "sequence 0: place 1"), ([3, 1], [0, 1, 3, 0, -1], "sequence 0: place 2"), ([1, 1], [-1, -1, -1, 0, -1], "sequence 0: place 0"),
    ([1, 2], [0, -1, -1, 0, -1], "sequence 1: place 1")])
def test_wrong_paths_are_reported_and_left_out(lengths, path, says):
    m = TreeModel(n_q=4, n_kv=2, d=64, batch=2)
    k0, ends = m.k.clone(), torch.zeros(2, dtype=torch.int32, device="cuda")
    m.keep([0, 3, 5], None, [10, 20], lengths, path, ends)
    with pytest.raises(M.MpkError, match=says) as e:
        m.status()
    assert e.value.status == M.MPK_ERR_DEVICE
    m.graph.reset()
    bad = int(says[9])
    assert ends.tolist() == [p if i == bad else p + n for i, (p, n) in enumerate(zip([10, 20], lengths))] and torch.equal(_bits(k0[:, bad]), _bits(m.k[:, bad]))


@pytest.mark.parametrize("bad", [-1, 50, 2 ** 31 - 1])
def test_a_page_outside_the_pool_is_reported_and_never_dereferenced(bad):
    m = TreeModel(n_q=4, n_kv=2, d=64, batch=2, max_seq=64, page=8, pages=50)
    m.table[1, 2] = bad
    parents = [-1, 0, 0, -1, 0, 1, 1, 2]
    x, q, o, work = m.normal(8, 8 * 64), m.normal(8, 256), m.normal(8, 256), workspace()
    args = ([0, 3, 8], None, [4, 15], parents)
    for call in (lambda: m.tree_append(0, *args, x, q), lambda: m.tree_attend(0, *args, q, o, work),
                 lambda: m.keep([0, 3, 8], None, [4, 15], [2, 3], [0, 2, -1, 0, 2, 4, -1, -1])):
        call()
        with pytest.raises(M.MpkError, match="sequence 1: a page-table entry"):
            m.status()
        m.graph.reset()
    want, bound = tree_attend_exact(q[:3].view(3, 4, 64), m.cached(m.k, 0, 0, 7), m.cached(m.v, 0, 0, 7), 4, parents[:3])
    # (keep has moved sequence 0's node 2 to place 1: its row is compared where nodes 0 and 1 only are seen)
    assert ((o[:1].view(1, 4, 64).double() - want[:1]).abs() <= bound[:1]).all()


def test_calls_of_no_rows_do_nothing():
    m = TreeModel(n_q=4, n_kv=2, d=64, batch=3)
    k0, b, p = m.k.clone(), m.ints([0, 0, 0, 0]), m.ints([1, 2, 3])
    s, ends = torch.cuda.current_stream().cuda_stream, m.ints([9, 9, 9])
    m.graph.tree_append(0, 3, 0, b.data_ptr(), 0, p.data_ptr(), 0, 0, 0, 0, 0, 0, s)
    m.graph.tree_attend(0, 3, 0, b.data_ptr(), 0, p.data_ptr(), 0, 0, 0, 0, 0, 0, s)
    m.graph.tree_keep(3, 0, b.data_ptr(), 0, p.data_ptr(), 0, 0, ends.data_ptr(), s)
    m.status()
    assert torch.equal(_bits(k0), _bits(m.k)) and ends.tolist() == [1, 2, 3]


def _rms(m, x, g):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + m.eps) * g.float()


def _layers(m, h, begin, slots, pos, parents, work):
    """Nodes through the layers of the model, the calls on trees for their part; logits."""
    for l, w in enumerate(m.w):
        qkv = _rms(m, h, w["attn_norm"]) @ w["wqkv"].float().t()
        q, o = (torch.empty(len(h), m.n_q * m.d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        m.tree_append(l, begin, slots, pos, parents, qkv, q)
        m.tree_attend(l, begin, slots, pos, parents, q, o, work)
        h = h + o.float() @ w["wo"].float().t()
        gate, up = (_rms(m, h, w["mlp_norm"]) @ w["wgu"].float().t()).chunk(2, -1)
        h = h + (torch.nn.functional.silu(gate) * up) @ w["wd"].float().t()
    return _rms(m, h, m.outer["final_norm"]) @ m.outer["lm_head"].float().t()


@pytest.mark.parametrize("kw", [dict(n_q=8, n_kv=2, d=64, qk_norm=True), dict(n_q=8, n_kv=2, d=128, page=16, pages=60, theta=1e6)])
def test_drafted_tokens_through_trees_equal_decoding_them(kw):
    """Two sequences decode greedily, token by token.  The same from trees: wrong guesses beside the tokens that the decoder found, three
    times; what is accepted, where the cache stands and what the next step says, all of it left in device memory, against the decoder."""
    kw = dict(kw, batch=2, vocab=64, layers=3, max_seq=192, seed=5)
    a, b = TreeModel(**kw), TreeModel(**kw)
    stream, lens, steps = torch.cuda.current_stream().cuda_stream, [37, 90], 16
    tok, pos = a.ints([3, 11]), a.ints(lens)
    tokens, logits = [tok.tolist()], []
    for _ in range(steps):
        lg = torch.empty(2, 64, device="cuda")
        a.graph.decode_step(tok.data_ptr(), pos.data_ptr(), lg.data_ptr(), stream)
        a.status()
        tok, pos = lg.argmax(-1).to(torch.int32), pos + 1
        tokens.append(tok.tolist())
        logits.append(lg)
    scale = max(float(x.abs().max()) for x in logits)
    # queries, probabilities and outputs of three layers in bf16: the decoder's are fp32
    far = 8 * BF16_HALF * scale
    done, work, rng = [0, 0], workspace(), random.Random(1)
    pos = b.ints(lens)
    for _ in range(3):
        # nodes: the last token, then per depth the decoder's token behind two wrong guesses, all children of its last one
        parents, guess, each = [], [], []
        for i in range(2):
            p, g, last = [-1], [tokens[done[i]][i]], 0
            for k in range(1, 5 if i else 4):
                right = tokens[done[i] + k][i] if k < 4 else (tokens[done[i] + k][i] + 1) % 64   # (the fifth level is wrong altogether)
                for j in range(3):
                    p.append(last)
                    g.append(right if j == 2 else (right + 1 + rng.randrange(62)) % 64)
                last = len(p) - 1
            parents.append(p)
            guess.append(g)
            each.append(len(p))
        begin = _begin(each)
        flat, ids = sum(parents, []), sum(guess, [])
        at = pos.tolist()
        lg = _layers(b, b.outer["embed"][torch.tensor(ids, device="cuda")].float(), begin, None, at, flat, work)
        lengths, path, nxt, lp = b.verify(begin, flat, ids, lg, work)
        ends = torch.empty(2, dtype=torch.int32, device="cuda")
        b.graph.tree_keep(2, begin[-1], b.ints(begin).data_ptr(), 0, pos.data_ptr(), lengths.data_ptr(), path.data_ptr(), ends.data_ptr(), stream)
        b.status()
        for i in range(2):
            n = int(lengths[i])
            walk = path[begin[i]:begin[i] + n].tolist()
            said = [ids[begin[i] + t] for t in walk[1:]] + [int(nxt[i])]
            for k, (t, x) in enumerate(zip(walk, said)):
                want = logits[done[i] + k][i]
                assert (lg[begin[i] + t] - want).abs().max() < far
                assert want[x] >= want.max() - 2 * far   # the decoder's token, or one as good as it
                assert abs(float(lp[begin[i] + k] - torch.log_softmax(lg[begin[i] + t].double(), -1)[x])) < 1e-5
            assert n == 4 and said == [tokens[done[i] + k][i] for k in range(1, 5)], "a near tie: other tokens from here on"
            done[i] += n
        pos = ends
    assert pos.tolist() == [n + d for n, d in zip(lens, done)]
    out = torch.empty(2, 64, device="cuda")
    b.graph.decode_step(nxt.data_ptr(), pos.data_ptr(), out.data_ptr(), stream)   # the graph decodes on
    b.status()
    assert torch.isfinite(out).all() and (out - logits[done[0]]).abs().max() < far


def test_captured_calls_follow_the_trees_of_each_replay():
    m = TreeModel(n_q=8, n_kv=2, d=64, max_seq=640, batch=3, layers=2, page=16, pages=140, vocab=500)
    rows = 256
    x, q, out = m.normal(rows, 12 * 64), torch.zeros(rows, 512, dtype=torch.bfloat16, device=m.dev), torch.zeros(rows, 512, dtype=torch.bfloat16, device=m.dev)
    logits = m.normal(rows, 500, dtype=torch.float32, std=3.0)
    begin, slots, pos, ends = m.ints([0, 0, 0, 0]), m.ints([0, 1, 2]), m.ints([0, 0, 0]), m.ints([0, 0, 0])
    parents, tokens, work = m.ints([-1] * rows), m.ints([0] * rows), workspace()
    heat, uniform = torch.tensor([0.0, 1.0, 0.7], device=m.dev), torch.rand(rows, device=m.dev)
    lengths, path, nxt, lp = m.ints([0] * 3), m.ints([0] * rows), m.ints([0] * 3), torch.zeros(rows, device=m.dev)

    def calls(stream):
        lists = (begin.data_ptr(), slots.data_ptr(), pos.data_ptr())
        m.graph.tree_append(0, 3, rows, *lists, parents.data_ptr(), x.data_ptr(), M.ROWS_BF16, x.stride(0), q.data_ptr(), q.stride(0), stream)
        m.graph.tree_attend(0, 3, rows, *lists, parents.data_ptr(), q.data_ptr(), q.stride(0), out.data_ptr(), out.stride(0), work.data_ptr(), stream)
        m.graph.tree_verify(3, rows, begin.data_ptr(), parents.data_ptr(), tokens.data_ptr(), logits.data_ptr(), M.ROWS_F32, 500, 0, 0, 0,
                            heat.data_ptr(), uniform.data_ptr(), lengths.data_ptr(), path.data_ptr(), nxt.data_ptr(), lp.data_ptr(), work.data_ptr(), stream)
        m.graph.tree_keep(3, rows, *lists, lengths.data_ptr(), path.data_ptr(), ends.data_ptr(), stream)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(torch.cuda.current_stream().cuda_stream)
    for n, (lens, p, s) in enumerate((([1, 1, 1], [300, 0, 77], [0, 1, 2]), ([200, 0, 56], [100, 600, 0], [2, 0, 1]), ([0, 0, 256], [0, 0, 384], [0, 1, 2]),
                                      ([3, 2, 4], [16, 630, 333], [1, 2, 0]), ([0, 0, 0], [0, 0, 0], [0, 1, 2]))):
        flat, each = _forest(lens, ["random"] * 3, behind=rows - sum(lens), seed=n)
        begin.copy_(m.ints(_begin(lens))), pos.copy_(m.ints(p)), slots.copy_(m.ints(s)), parents.copy_(m.ints(flat))
        tokens.copy_(logits.argmax(-1).roll(1).to(torch.int32)), uniform.copy_(torch.rand(rows, device=m.dev))
        k0, v0 = m.k.clone(), m.v.clone()
        everything = (q, out, lengths, path, nxt, lp, ends, m.k, m.v)
        for t in everything[:-2]:
            t.fill_(7)
        graph.replay()
        m.status()
        got = [t.clone() for t in everything]
        assert (got[1][sum(lens):] == 7).all() and (got[3][sum(lens):] == 7).all() and (got[5][sum(lens):] == 7).all()
        m.k.copy_(k0), m.v.copy_(v0)
        for t in everything[:-2]:
            t.fill_(7)
        calls(torch.cuda.current_stream().cuda_stream)
        m.status()
        for t, g in zip(everything, got):
            assert torch.equal(t.view(torch.int16) if t.dtype == torch.bfloat16 else t, g.view(torch.int16) if g.dtype == torch.bfloat16 else g)
        assert torch.equal(got[6], pos + got[2])


def test_the_same_call_gives_the_same_bits_on_any_stream():
    m, lens, pos, slots, begin, parents, each, q = _attend_case(ATTEND[12])
    outs, work = [], workspace()
    torch.cuda.synchronize()
    for i in range(4):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            out = torch.zeros(q.shape[0], m.n_q * m.d, dtype=torch.bfloat16, device="cuda")
            m.tree_attend(0, begin, slots, pos, parents, q, out, work)
        stream.synchronize()
        outs.append(out)
    m.status()
    assert all(torch.equal(_bits(o), _bits(outs[0])) for o in outs)


def test_a_graph_with_fewer_slots_than_its_cache_has():
    """As a graph of a set: the same calls through a graph of two sequences on the cache of one of five leave the same bits in every layer."""
    m = TreeModel(n_q=8, n_kv=2, d=64, batch=5, max_seq=512, layers=3)
    ptrs = {n: t.data_ptr() for n, t in m.outer.items()}
    ptrs["layers"] = [{n: t.data_ptr() for n, t in lw.items()} for lw in m.w]
    shape, whole = SimpleNamespace(**dict(vars(m.shape), batch=2)), m.graph
    part = M.compile_graph(shape, ptrs, (m.k.data_ptr(), m.v.data_ptr()), fusion=31, transitive_reduction=1, kv_batch=5)
    lens, pos, begin, work = [90, 40], [300, 17], [0, 90, 130], workspace()
    flat, _ = _forest(lens, ["random"] * 2, seed=3)
    x, k0, v0, got = m.normal(130, 12 * 64), m.k.clone(), m.v.clone(), []
    path, lengths = [0, 2, 50, 89] + [-1] * 86 + [1, 39] + [-1] * 38, [4, 2]
    for graph in (whole, part):
        m.graph = graph
        m.k.copy_(k0), m.v.copy_(v0)
        outs = []
        for layer in range(3):
            q, out = (torch.zeros(130, 512, dtype=torch.bfloat16, device=m.dev) for _ in range(2))
            m.tree_append(layer, begin, [1, 0], pos, flat, x, q)
            m.tree_attend(layer, begin, [1, 0], pos, flat, q, out, work)
            outs += [q, out]
        m.keep(begin, [1, 0], pos, lengths, path)
        m.status()
        got.append(outs + [m.k.clone(), m.v.clone()])
    assert all(torch.equal(_bits(a), _bits(b)) for a, b in zip(*got))
    assert not torch.equal(_bits(got[0][-1]), _bits(v0))
