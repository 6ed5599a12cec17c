"""Trees of drafted tokens on a graph's cache, measured: filling the cache with the nodes of several trees
(`Graph.tree_append`), their attention over the cache and their ancestors (`Graph.tree_attend`), the walk that
accepts or rejects them by the target's logits and given random numbers (`Graph.tree_verify`), and closing up the
cache rows of what was accepted (`Graph.tree_keep`).

A case is one call of one of them: a program that drafts ahead makes the first two once a layer, the others once a
step.  With `own` false the same results come from elementary torch operations, in 32 bits; angles, and everything
that a random number is compared with, in 64.

Queries, keys and values are N(0, 1), gains 1 + N(0, 0.02), as in the repository's synthetic models.  Logits are
N(0, 2.5) with drafted and other tokens raised, so that about seven of ten nodes have a child that is accepted.
"""
import math
import random
from types import SimpleNamespace

import torch

import paper_2512_22219_amd as M

own = False
EPS = 1e-6
ACCEPT = 0.7   # of a node with children, about: that one of them is accepted


def _case(name, op, **kw):
    # nodes: rows of a sequence's tree, cached: rows in front of it, from .. to over the sequences; depth, fan: no node
    # has more ancestors, no node more children
    c = dict(op=op, seqs=1, nodes_lo=1, nodes_hi=1, depth=6, fan=4)
    if op == "verify":
        # draft: "none" (tokens chosen), "drawn" (from a distribution, independently), "once" (without replacement)
        c.update(vocab=151936, type="f32", temperature=1.0, draft="none")
    else:
        c.update(q_heads=32, kv_heads=8, head_dim=128, theta=1e6, qk_norm=False, cached_lo=0, cached_hi=0, page=0, type="bf16")
    if op == "keep":
        c.update(layers=1, kept_lo=1, kept_hi=1)   # nodes on the accepted path
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest call: a few drafted tokens of one request, the 8B shape with the query/key norm; nothing but latency
        _case("append 8 nodes", "append", nodes_lo=8, nodes_hi=8, qk_norm=True, cached_lo=1024, cached_hi=1024),
        # a full batch's trees on the serving cache, fp32 projections, 70B heads
        _case("append 16 x 64 nodes, paged", "append", seqs=16, nodes_lo=64, nodes_hi=64, q_heads=64, theta=5e5, cached_lo=100,
              cached_hi=3000, page=16, type="f32"),
        # one request's small tree over the benchmark's cache: a short call
        _case("attend 8 nodes over 1024", "attend", nodes_lo=8, nodes_hi=8, cached_lo=1024, cached_hi=1024),
        # eight requests with the benchmark's ragged cache lengths, trees of odd sizes: all memory
        _case("attend 8 ragged trees", "attend", seqs=8, nodes_lo=9, nodes_hi=41, theta=5e5, cached_lo=512, cached_hi=4096),
        # one tree over a long cache, head size 64, pages of 16: split over the long axis
        _case("attend 64 nodes over 30000, paged", "attend", nodes_lo=64, nodes_hi=64, depth=10, head_dim=64, cached_lo=30001,
              cached_hi=30001, page=16),
        # the largest: four trees of 256 nodes behind long caches on the 70B shape
        _case("attend 4 x 256 nodes over 12000", "attend", seqs=4, nodes_lo=256, nodes_hi=256, depth=12, q_heads=64, theta=5e5,
              cached_lo=11000, cached_hi=12000),
        # one request, greedy: a chain of five drafted tokens behind the last one
        _case("verify a chain of 6, greedy", "verify", nodes_lo=6, nodes_hi=6, depth=5, fan=1, temperature=0.0),
        # one request, sampled, the tree's tokens chosen by rank
        _case("verify 64 nodes", "verify", nodes_lo=64, nodes_hi=64),
        # a full batch, sampled, tokens drawn from the draft's distribution without replacement, logits in bf16
        _case("verify 8 x 25 nodes, drawn", "verify", seqs=8, nodes_lo=25, nodes_hi=25, vocab=128256, type="bf16", temperature=0.8,
              draft="once"),
        # the largest: a full batch's trees
        _case("verify 16 x 64 nodes", "verify", seqs=16, nodes_lo=64, nodes_hi=64, temperature=0.8),
        # one request of the 8B shape, four drafted tokens accepted
        _case("keep 5 of 32 nodes", "keep", nodes_lo=32, nodes_hi=32, layers=36, kept_lo=5, kept_hi=5, cached_lo=300, cached_hi=300),
        # a full batch on the serving cache
        _case("keep 16 paths, paged", "keep", seqs=16, nodes_lo=20, nodes_hi=64, layers=32, kept_lo=1, kept_hi=9, cached_lo=10,
              cached_hi=200, page=16),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "verify", "verify", "keep"])
    c = _case(None, op, seqs=rng.choice([1, 1, 2, 3, 5, 8, 13, 16]), depth=rng.choice([1, 3, 5, 8, 20]), fan=rng.choice([1, 2, 4, 10]))
    c["nodes_hi"] = _log(rng, 1, min(256, 1024 // c["seqs"]))
    c["nodes_lo"] = rng.choice([c["nodes_hi"], rng.randint(1, c["nodes_hi"])])
    if op == "verify":
        c.update(vocab=_log(rng, 1000, 152000), type=rng.choice(["f32", "bf16"]), temperature=rng.choice([0.0, 0.6, 0.8, 1.0, 1.0]),
                 draft=rng.choice(["none", "none", "drawn", "once"]))
        most = ((1 << 27) if c["draft"] == "none" else (1 << 25)) // c["vocab"] // c["seqs"]
        c["nodes_hi"] = max(1, min(c["nodes_hi"], most))
        c["nodes_lo"] = min(c["nodes_lo"], c["nodes_hi"])
        return c
    c.update(head_dim=rng.choice([64, 128]), theta=rng.choice([1e4, 5e5, 1e6]), qk_norm=rng.random() < 0.5,
             page=rng.choice([0, 0, 8, 16, 64]))
    c["kv_heads"] = rng.choice([2, 4, 8])
    c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 8])
    c["cached_hi"] = _log(rng, 1, (6000 if op == "keep" else 48000) // c["seqs"]) - 1
    c["cached_lo"] = rng.choice([0, c["cached_hi"], rng.randint(0, c["cached_hi"])])
    if op == "append":
        c["type"] = rng.choice(["bf16", "f32"])
    if op == "attend":
        while c["seqs"] * c["q_heads"] * c["nodes_hi"] * (c["cached_hi"] + c["nodes_hi"]) > 3 << 28:   # (the plain form's scores)
            c["cached_hi"] = c["cached_hi"] // 2
            c["cached_lo"] = min(c["cached_lo"], c["cached_hi"])
    if op == "keep":
        c["layers"] = rng.randint(1, 36)
        c["kept_hi"] = rng.randint(1, min(16, (c["nodes_lo"] + 1) // 2))
        c["kept_lo"] = rng.randint(1, c["kept_hi"])
    return c


def _spread(n, lo, hi, step):
    return [hi - (hi - lo) * (i * step % n) // max(1, n - 1) for i in range(n)]


def _lens(c):
    """(nodes, rows cached before) of every sequence: spread over their ranges, in a mixed order, the largest first."""
    n = c["seqs"]
    odd = next(s for s in (5, 7, 11) if n % s)
    return _spread(n, c["nodes_lo"], c["nodes_hi"], 1), _spread(n, c.get("cached_lo", 0), c.get("cached_hi", 0), odd)


def _kept(c):
    return _spread(c["seqs"], c["kept_lo"], c["kept_hi"], next(s for s in (3, 5, 7) if c["seqs"] % s))


def _tree(rng, nodes, depth, fan):
    """Parents of a tree of at most that depth and fan; what has no room in one is a chain behind its last node."""
    parents, deep, kids, open_ = [-1], [0], [0], [0]
    while len(parents) < nodes:
        room = [t for t in open_ if deep[t] < depth and kids[t] < fan]
        if not room:
            room = [len(parents) - 1]
        p = room[min(int(len(room) * rng.random() ** 2), len(room) - 1)]
        kids[p] += 1
        parents.append(p)
        deep.append(deep[p] + 1)
        kids.append(0)
        open_ = room + [len(parents) - 1]
    return parents


def _deepest(c):
    """The depth that no node is below: the case's, or that of a chain where its nodes do not fit its depth and fan."""
    room, width = 0, 1
    for _ in range(c["depth"] + 1):
        room, width = room + width, min(width * c["fan"], 256)
        if room >= c["nodes_hi"]:
            return min(c["depth"], c["nodes_hi"] - 1)
    return c["nodes_hi"] - 1


# ---------------------------------------------------------------------------------- inputs
def _normal(gen, *size, std=1.0, dtype=torch.bfloat16):
    return torch.empty(size, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def _inputs(c, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    rng = random.Random(seed)
    nodes, cached = _lens(c)
    n, rows = c["seqs"], sum(nodes)
    trees = [_tree(rng, t, c["depth"], c["fan"]) for t in nodes]
    begin = [sum(nodes[:i]) for i in range(n + 1)]
    inp = {"rows": rows, "longest": max(nodes), "begin": begin, "trees": trees, "deepest": _deepest(c)}
    inp["row_begin"] = torch.tensor(begin, dtype=torch.int32, device=dev)
    inp["parents"] = torch.tensor(sum(trees, []), dtype=torch.int32, device=dev)
    if c["op"] == "verify":
        return _verify_inputs(c, inp, gen, rng)
    nkv, d = c["kv_heads"], c["head_dim"]
    step = c["page"] or 8
    max_seq = -(-max(a + b for a, b in zip(nodes, cached)) // step) * step
    inp.update(max_seq=max_seq, pages=0, positions=torch.tensor(cached, dtype=torch.int32, device=dev))
    layers = c.get("layers", 1)
    if c["page"]:   # every sequence's blocks in pages of a shuffled pool
        blocks = max_seq // c["page"]
        inp["pages"] = n * blocks + 3
        deal = torch.randperm(inp["pages"], generator=gen, device=dev)
        inp["table"] = deal[: n * blocks].view(n, blocks).to(torch.int32)
        size = (layers, inp["pages"], nkv, c["page"], d)
    else:
        size = (layers, n, nkv, max_seq, d)
    inp["k"], inp["v"] = _normal(gen, *size), _normal(gen, *size)
    if c["op"] == "keep":
        # paths that leave some first nodes where they are, then nodes behind all the places that are filled, so that a
        # pass on the rows that a pass has left does the same again
        kept, path = _kept(c), []
        for t, k in zip(nodes, kept):
            k = min(k, (t + 1) // 2)
            stay = rng.randint(1, k)
            p = list(range(stay)) + sorted(rng.sample(range(k, t), k - stay))
            path.append(p + [-1] * (t - k))
        inp["paths"] = path
        inp["path"] = torch.tensor(sum(path, []), dtype=torch.int32, device=dev)
        inp["lengths"] = torch.tensor([sum(x >= 0 for x in p) for p in path], dtype=torch.int32, device=dev)
        inp["most"] = max(kept)
        return inp
    heads = c["q_heads"] + (2 * nkv if c["op"] == "append" else 0)
    inp["x"] = _normal(gen, rows, heads * d, dtype=torch.float32 if c["type"] == "f32" else torch.bfloat16)
    for g in ("q_norm", "k_norm"):
        inp[g] = (1.0 + _normal(gen, d, std=0.02, dtype=torch.float32)).to(torch.bfloat16)
    inp["inv_freq"] = c["theta"] ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=dev) / d)
    return inp


def _verify_inputs(c, inp, gen, rng):
    dev, V, rows, temp = torch.device("cuda"), c["vocab"], inp["rows"], c["temperature"]
    x = _normal(gen, rows, V, std=2.5, dtype=torch.float32)
    up = torch.randint(V, (rows,), generator=gen, device=dev)   # a token that the draft does not know of
    tokens = torch.randint(V, (rows,), generator=gen, device=dev)
    inp["uniforms"] = torch.rand(rows, generator=gen, device=dev)
    inp["temperatures"] = torch.full((c["seqs"],), temp, device=dev)
    inp["draft"] = None
    if c["draft"] == "none":   # chosen by rank: the first child the likeliest, more mass on the children than elsewhere
        tau = temp or 1.0
        total = math.log(V) + (2.5 / tau) ** 2 / 2
        first, at, height = 0, [[], []], []
        for tree in inp["trees"]:
            kids = {}
            for t, p in enumerate(tree):
                if p < 0:
                    continue
                j = kids[p] = kids.get(p, 0) + 1
                at[0].append(first + p)
                at[1].append(first + t)
                height.append(tau * (total + math.log(1.6 * rng.uniform(0.5, 1.5) / j ** 1.5)))
            first += len(tree)
        if height:
            at = torch.tensor(at, device=dev)
            x.view(-1).scatter_(0, at[0] * V + tokens[at[1]], torch.tensor(height, device=dev))
        if temp == 0:   # three in ten rows have another arg max than the drafted tokens
            over = (torch.rand(rows, generator=gen, device=dev) > ACCEPT).float() * (total + 5)
            x.scatter_add_(1, up[:, None], over[:, None])
    else:   # drawn: the draft's logits are the target's with an error
        x.scatter_add_(1, up[:, None], 15 * torch.rand(rows, 1, generator=gen, device=dev))
        tau = temp or 1.0
        inp["draft"] = torch.softmax((x + 0.7 * torch.empty_like(x).normal_(generator=gen)) / tau, 1)
        race = inp["draft"] / torch.empty_like(x).exponential_(generator=gen)
        first = 0
        kids_most = max([tree.count(p) for tree in inp["trees"] for p in set(tree) - {-1}], default=0)
        best = race.topk(kids_most, 1).indices if kids_most else None   # the race's first, second, ..: drawn without replacement
        place = [[], [], []]
        for tree in inp["trees"]:
            kids = {}
            for t, p in enumerate(tree):
                if p < 0:
                    continue
                place[0].append(first + t)
                place[1].append(first + p)
                place[2].append(kids.get(p, 0))
                kids[p] = kids.get(p, 0) + 1
            first += len(tree)
        if place[0]:
            t, p, j = (torch.tensor(y, device=dev) for y in place)
            if c["draft"] == "drawn":
                tokens[t] = torch.multinomial(inp["draft"], kids_most, replacement=True, generator=gen)[p, j]
            else:
                tokens[t] = best[p, j]
    inp["tokens"] = tokens.to(torch.int32)
    inp["logits"] = x.to(torch.float32 if c["type"] == "f32" else torch.bfloat16)
    return inp


def _graph(c, inp):
    """The compiled graph that the calls belong to: small layers of the case's heads, over the case's cache."""
    dev, bf = torch.device("cuda"), torch.bfloat16
    verify = c["op"] == "verify"
    nq, nkv, d = (4, 2, 64) if verify else (c["q_heads"], c["kv_heads"], c["head_dim"])
    H, F, V = 128, 256, c["vocab"] if verify else 1024
    max_seq, layers = 64 if verify else inp["max_seq"], c.get("layers", 1)
    norm = not verify and c["qk_norm"]
    shape = SimpleNamespace(n_layers=layers, hidden=H, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, ffn=F, vocab=V, rms_eps=EPS,
                            rope_theta=1e4 if verify else c["theta"], batch=c["seqs"], max_seq=max_seq, n_experts=0, top_k=0,
                            expert_ffn=0, qk_norm=norm)

    def zeros(*size):
        return torch.zeros(size, dtype=bf, device=dev)

    w = {"attn_norm": zeros(H), "wqkv": zeros((nq + 2 * nkv) * d, H), "wo": zeros(H, nq * d), "mlp_norm": zeros(H),
         "wgu": zeros(2 * F, H), "wd": zeros(H, F)}
    if norm:
        gain = inp.get("q_norm", w["attn_norm"][:d])
        w.update(q_norm=gain, k_norm=inp.get("k_norm", gain))
    outer = {"embed": zeros(V, H), "final_norm": zeros(H), "lm_head": zeros(V, H)}
    k, v = (zeros(1, c["seqs"], nkv, max_seq, d), zeros(1, c["seqs"], nkv, max_seq, d)) if verify else (inp["k"], inp["v"])
    ptrs = {n: t.data_ptr() for n, t in outer.items()}
    ptrs["layers"] = [{n: t.data_ptr() for n, t in w.items()}] * layers
    paged = {} if verify or not c["page"] else dict(kv_page_size=c["page"], kv_pages=inp["pages"])
    graph = M.compile_graph(shape, ptrs, (k.data_ptr(), v.data_ptr()), fusion=31, transitive_reduction=1, **paged)
    if paged:
        graph.set_page_table(inp["table"].data_ptr())
    return graph, (w, outer, k, v)


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    st = {"case": c, "inputs": _inputs(c, seed)}
    inp = st["inputs"]
    st["graph"], st["weights"] = _graph(c, inp)
    st["work"] = torch.empty(96 << 20, dtype=torch.uint8, device=dev)
    if c["op"] in ("verify", "keep"):
        st["lengths"], st["next"] = (torch.empty(c["seqs"], dtype=torch.int32, device=dev) for _ in range(2))
        st["path"] = torch.empty(inp["rows"], dtype=torch.int32, device=dev)
        st["logprobs"] = torch.empty(inp["rows"], dtype=torch.float32, device=dev)
    else:
        st["out"] = torch.empty((inp["rows"], c["q_heads"] * c["head_dim"]), dtype=torch.bfloat16, device=dev)
    torch.cuda.synchronize()
    return st


# ---------------------------------------------------------------------------------- one pass
def run(st):
    return (OWN if own else PLAIN)[st["case"]["op"]](st)


def _own_append(st):
    c, inp, g = st["case"], st["inputs"], st["graph"]
    g.tree_append(0, c["seqs"], inp["rows"], inp["row_begin"].data_ptr(), 0, inp["positions"].data_ptr(), inp["parents"].data_ptr(),
                  inp["x"].data_ptr(), M.ROWS_F32 if c["type"] == "f32" else M.ROWS_BF16, inp["x"].stride(0), st["out"].data_ptr(),
                  st["out"].stride(0), torch.cuda.current_stream().cuda_stream)
    return [st["out"], inp["k"], inp["v"]]


def _own_attend(st):
    c, inp, g = st["case"], st["inputs"], st["graph"]
    g.tree_attend(0, c["seqs"], inp["rows"], inp["row_begin"].data_ptr(), 0, inp["positions"].data_ptr(), inp["parents"].data_ptr(),
                  inp["x"].data_ptr(), inp["x"].stride(0), st["out"].data_ptr(), st["out"].stride(0), st["work"].data_ptr(),
                  torch.cuda.current_stream().cuda_stream)
    return [st["out"]]


def _own_verify(st):
    c, inp, g = st["case"], st["inputs"], st["graph"]
    x, q = inp["logits"], inp["draft"]
    g.tree_verify(c["seqs"], inp["rows"], inp["row_begin"].data_ptr(), inp["parents"].data_ptr(), inp["tokens"].data_ptr(), x.data_ptr(),
                  M.ROWS_F32 if c["type"] == "f32" else M.ROWS_BF16, x.stride(0), 0 if q is None else q.data_ptr(),
                  0 if q is None else q.stride(0), M.TREE_DRAWN_ONCE if c["draft"] == "once" else 0, inp["temperatures"].data_ptr(),
                  inp["uniforms"].data_ptr(), st["lengths"].data_ptr(), st["path"].data_ptr(), st["next"].data_ptr(), st["logprobs"].data_ptr(),
                  st["work"].data_ptr(), torch.cuda.current_stream().cuda_stream)
    return [st["lengths"], st["path"], st["next"], st["logprobs"]]


def _own_keep(st):
    c, inp, g = st["case"], st["inputs"], st["graph"]
    g.tree_keep(c["seqs"], inp["rows"], inp["row_begin"].data_ptr(), 0, inp["positions"].data_ptr(), inp["lengths"].data_ptr(),
                inp["path"].data_ptr(), st["next"].data_ptr(), torch.cuda.current_stream().cuda_stream)
    return [st["next"], inp["k"], inp["v"]]


OWN = dict(append=_own_append, attend=_own_attend, verify=_own_verify, keep=_own_keep)


def _row_places(inp):
    """The sequence of every row and its place in the sequence."""
    r = torch.arange(inp["rows"], device=inp["row_begin"].device)
    seq = (r[:, None] >= inp["row_begin"][None, 1:]).sum(1)
    return seq, r - inp["row_begin"][seq]


def _padded(inp, x, fill):
    """Rows' values as [sequence][longest], `fill` where a sequence has no row."""
    T = inp["longest"]
    t = torch.arange(T, device=x.device)
    size = (inp["row_begin"][1:] - inp["row_begin"][:-1])[:, None]
    at = (inp["row_begin"][:-1, None] + t).clamp(max=inp["rows"] - 1)
    return torch.where(t < size, x[at], fill)


def _ancestors(inp):
    """[sequence][node][node]: is the second the first or an ancestor of it."""
    T = inp["longest"]
    t = torch.arange(T, device=inp["parents"].device)
    parent = (_padded(inp, inp["parents"], -1)[..., None] == t).float()
    own_, seen = torch.eye(T, device=t.device), torch.eye(T, device=t.device).expand(parent.shape)
    for _ in range(inp["deepest"]):
        seen = torch.matmul(parent, seen) + own_
    return seen > 0


def _plain_append(st):
    c, inp = st["case"], st["inputs"]
    nq, nkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    x = inp["x"].float().view(inp["rows"], nq + 2 * nkv, d)
    q, k, v = x.split((nq, nkv, nkv), 1)
    if c["qk_norm"]:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + EPS) * inp["q_norm"].float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + EPS) * inp["k_norm"].float()
    seq, t = _row_places(inp)
    depth = _ancestors(inp).sum(-1)[seq, t] - 1
    angle = (inp["positions"][seq] + depth).double()[:, None] * inp["inv_freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = torch.cat([q, k], 1)
    lo, hi = x[..., : d // 2], x[..., d // 2:]
    x = torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).to(torch.bfloat16)
    row = inp["positions"][seq] + t
    at = seq
    if c["page"]:
        at, row = inp["table"][seq, row // c["page"]].long(), row % c["page"]
    inp["k"][0][at, :, row] = x[:, nq:]
    inp["v"][0][at, :, row] = v.to(torch.bfloat16)
    return [x[:, :nq].reshape(inp["rows"], nq * d), inp["k"], inp["v"]]


def _plain_attend(st):
    c, inp = st["case"], st["inputs"]
    nq, nkv, d, n = c["q_heads"], c["kv_heads"], c["head_dim"], c["seqs"]
    G, T, S = nq // nkv, inp["longest"], inp["max_seq"]
    k, v = inp["k"][0], inp["v"][0]
    if c["page"]:
        k, v = (x[inp["table"].long()].transpose(1, 2).reshape(n, nkv, S, d) for x in (k, v))
    t = torch.arange(T, device=k.device)
    rows = (inp["row_begin"][:-1, None] + t).clamp(max=inp["rows"] - 1)
    q = inp["x"].float()[rows].view(n, T, nkv, G, d).permute(0, 2, 3, 1, 4).reshape(n, nkv, G * T, d)
    s = torch.matmul(q, k.float().transpose(2, 3).contiguous()).view(n, nkv, G, T, S)
    # what a node sees: the cached rows, itself and its ancestors
    place = torch.arange(S, device=k.device) - inp["positions"][:, None]
    near = _ancestors(inp).gather(2, place.clamp(0, T - 1)[:, None].expand(n, T, S))
    seen = (place < 0)[:, None] | (near & (place < T)[:, None])
    s = (s * d ** -0.5).masked_fill(~seen[:, None, None], -math.inf)
    s = (s - s.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(s.view(n, nkv, G * T, S), v.float()).view(n, nkv, G, T, d) / s.sum(-1, keepdim=True)
    seq, t = _row_places(inp)
    return [o.permute(0, 3, 1, 2, 4)[seq, t].reshape(inp["rows"], nq * d).to(torch.bfloat16)]


def _plain_verify(st):
    c, inp = st["case"], st["inputs"]
    n, T, dev = c["seqs"], inp["longest"], inp["parents"].device
    greedy = c["temperature"] == 0
    parents, tokens, uniform = (_padded(inp, inp[x], fill) for x, fill in (("parents", -2), ("tokens", -1), ("uniforms", 0.0)))
    tokens, uniform = tokens.long(), uniform.double()
    t, seqs = torch.arange(T, device=dev), torch.arange(n, device=dev)
    at, going = torch.zeros(n, dtype=torch.long, device=dev), torch.ones(n, dtype=torch.bool, device=dev)
    lengths, path = torch.zeros(n, dtype=torch.int32, device=dev), torch.full((n, T), -1, dtype=torch.int32, device=dev)
    left = torch.zeros(n, c["vocab"], dtype=torch.float64, device=dev)   # what the next token is drawn from
    logp, last = torch.zeros(n, T, dtype=torch.float64, device=dev), torch.zeros_like(left)
    best = torch.zeros(n, dtype=torch.long, device=dev)
    for level in range(inp["deepest"] + 1):
        path[:, level] = torch.where(going, at, -1).to(torch.int32)
        lengths += going
        row = inp["row_begin"][:-1] + at
        x = inp["logits"][row].double()
        top = torch.where(x == x.amax(1, keepdim=True), torch.arange(c["vocab"], device=dev), c["vocab"]).amin(1)
        best = torch.where(going, top, best)
        if not greedy:
            x = x / inp["temperatures"].double()[:, None]
        x = x - x.amax(1, keepdim=True)
        x = x - x.exp().sum(1, keepdim=True).log()
        r = x.exp()
        child = parents == at[:, None]
        order = child.cumsum(1)
        taken = torch.full((n,), -1, dtype=torch.long, device=dev)
        drawn = torch.zeros(n, dtype=torch.float64, device=dev)
        q = inp["draft"][row].double() if inp["draft"] is not None and not greedy else None
        for j in range(1, min(c["fan"], T - 1) + 1):
            hit = child & (order == j)
            some = hit.any(1) & (taken < 0)
            node = (hit * t).sum(1)
            token = tokens[seqs, node].clamp(min=0)
            if greedy:
                taken = torch.where(some & (token == top), node, taken)
                continue
            if q is None:
                share, less = 1.0, torch.zeros_like(r).scatter_(1, token[:, None], 2.0)
            else:
                scale = 1.0 / (1.0 - drawn) if c["draft"] == "once" else torch.ones_like(drawn)
                share = q.gather(1, token[:, None])[:, 0]
                drawn, less, share = drawn + share, q * scale[:, None], share * scale
            yes = some & (uniform[seqs, node] * share < r.gather(1, token[:, None])[:, 0])
            taken = torch.where(yes, node, taken)
            rest = (r - less).clamp(min=0)
            r = torch.where((some & ~yes)[:, None], rest / rest.sum(1, keepdim=True), r)
        left = torch.where((going & (taken < 0))[:, None], r, left)
        last = torch.where((going & (taken < 0))[:, None], x, last)
        going = going & (taken >= 0)
        logp[:, level] = torch.where(going, x.gather(1, tokens[seqs, taken][:, None].clamp(min=0))[:, 0], 0.0)
        at = torch.where(going, taken, at)
    if greedy:
        token = best
    else:
        below = left.cumsum(1)
        token = (below <= uniform[:, :1] * below[:, -1:]).sum(1)
    logp.scatter_add_(1, lengths[:, None].long() - 1, last.gather(1, token[:, None]))
    seq, t = _row_places(inp)
    return [lengths, path[seq, t], token.to(torch.int32), logp[seq, t].float()]


def _plain_keep(st):
    c, inp = st["case"], st["inputs"]
    n, most = c["seqs"], min(inp["most"], inp["longest"])
    path = _padded(inp, inp["path"], -1)[:, :most].long()
    keep = (torch.arange(most, device=path.device) < inp["lengths"][:, None]).nonzero(as_tuple=True)
    seq, place = keep
    source, target = inp["positions"][seq] + path[seq, place], inp["positions"][seq] + place
    for x in (inp["k"], inp["v"]):
        if c["page"]:
            x[:, inp["table"][seq, target // c["page"]].long(), :, target % c["page"]] = \
                x[:, inp["table"][seq, source // c["page"]].long(), :, source % c["page"]]
        else:
            x[:, seq, :, target] = x[:, seq, :, source]
    return [inp["positions"] + inp["lengths"], inp["k"], inp["v"]]


PLAIN = dict(append=_plain_append, attend=_plain_attend, verify=_plain_verify, keep=_plain_keep)


# ---------------------------------------------------------------------------------- what a pass needs
def work(case):
    c = case
    nodes, cached = _lens(c)
    if c["op"] == "verify":   # the rows of the nodes that the walk comes to
        deep = min(c["depth"], c["nodes_hi"] - 1)
        rows = c["seqs"] * sum(ACCEPT ** k for k in range(deep + 1))
        size = (4 if c["type"] == "f32" else 2) + (4 if c["draft"] != "none" and c["temperature"] else 0)
        return {"bytes": rows * c["vocab"] * size, "flops": 10.0 * rows * c["vocab"]}
    nq, nkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    if c["op"] == "keep":
        values = sum((k - 1) / 2 for k in _kept(c)) * c["layers"] * 2 * nkv * d   # (half of the paths, about, stays where it is)
        return {"bytes": 4.0 * values + 4.0 * sum(nodes) + 12.0 * c["seqs"], "flops": 0.0}
    if c["op"] == "append":
        values = sum(nodes) * (nq + 2 * nkv) * d
        return {"bytes": float(values * ((4 if c["type"] == "f32" else 2) + 2)), "flops": 10.0 * values}
    pairs = sum(t * (p + min(c["depth"], t) / 2 + 1) for t, p in zip(nodes, cached))
    return {"bytes": 4.0 * (sum(nodes) * nq * d + sum(t + p for t, p in zip(nodes, cached)) * nkv * d), "flops": 4.0 * pairs * nq * d}


# ---------------------------------------------------------------------------------- 64-bit results
def exact(case, seed):
    c, inp = case, _inputs(case, seed)
    nodes, cached = _lens(c)
    chains = []   # per sequence and node: the node and its ancestors, the root first
    for tree in inp["trees"]:
        chains.append([])
        for t, p in enumerate(tree):
            chains[-1].append((chains[-1][p] if p >= 0 else []) + [t])
    return EXACT[c["op"]](c, inp, nodes, cached, chains)


def _at(c, inp, x, i, rows):
    """The rows of a sequence's cache (of every layer): [layers][rows][kv heads][d]."""
    if c["page"]:
        return x[:, inp["table"][i].long()[rows // c["page"]], :, rows % c["page"]].transpose(0, 1)
    return x[:, i, :, rows].transpose(1, 2)


def _put(c, inp, x, i, rows, values):
    if c["page"]:
        x[:, inp["table"][i].long()[rows // c["page"]], :, rows % c["page"]] = values.transpose(0, 1)
    else:
        x[:, i, :, rows] = values.transpose(1, 2)


def _exact_append(c, inp, nodes, cached, chains):
    nq, nkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    k, v, out, first = inp["k"].double(), inp["v"].double(), [], 0
    for i, (T, p) in enumerate(zip(nodes, cached)):
        x = inp["x"][first:first + T].double().view(T, nq + 2 * nkv, d)
        q, kk, vv = x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:]
        if c["qk_norm"]:
            q, kk = (y / torch.sqrt((y * y).sum(-1, keepdim=True) / d + EPS) * inp[g].double() for y, g in ((q, "q_norm"), (kk, "k_norm")))
        where = torch.tensor([p + len(a) - 1 for a in chains[i]], dtype=torch.float64, device=x.device)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), where[:, None] * inp["inv_freq"])[:, None]
        q, kk = (torch.cat([z.real, z.imag], -1) for z in
                 (torch.complex(y[..., : d // 2].contiguous(), y[..., d // 2:].contiguous()) * turn for y in (q, kk)))
        out.append(q.reshape(T, nq * d))
        rows = torch.arange(p, p + T, device=x.device)
        _put(c, inp, k, i, rows, kk[None])
        _put(c, inp, v, i, rows, vv[None])
        first += T
    return [torch.cat(out), k, v]


def _exact_attend(c, inp, nodes, cached, chains):
    nq, nkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    out, first = [], 0
    for i, (T, p) in enumerate(zip(nodes, cached)):
        q = inp["x"][first:first + T].double().view(T, nkv, nq // nkv, d)
        rows = torch.arange(p + T, device=q.device)
        hidden = torch.ones(T, p + T, dtype=torch.bool)
        hidden[:, :p] = False
        for t, chain in enumerate(chains[i]):
            hidden[t, [p + a for a in chain]] = False
        hidden = hidden.to(q.device)
        kk, vv = (_at(c, inp, x, i, rows)[0].double() for x in (inp["k"], inp["v"]))
        o = torch.empty_like(q)
        for h in range(nkv):
            for g in range(nq // nkv):
                s = (q[:, h, g] @ kk[:, h].t() / math.sqrt(d)).masked_fill(hidden, -math.inf)
                o[:, h, g] = torch.softmax(s, -1) @ vv[:, h]
        out.append(o.reshape(T, nq * d))
        first += T
    return [torch.cat(out)]


def _exact_verify(c, inp, nodes, cached, chains):
    tokens, uniform = inp["tokens"].tolist(), inp["uniforms"].tolist()
    lengths, path, following, logs = [], [], [], []
    for i, tree in enumerate(inp["trees"]):
        first, at, walk, log = inp["begin"][i], 0, [], []
        while True:
            walk.append(at)
            x = inp["logits"][first + at].double()
            kids, onward = [t for t, p in enumerate(tree) if p == at], None
            p = torch.log_softmax(x / (float(inp["temperatures"][i]) or 1.0), 0)
            if c["temperature"] == 0:
                token = int((x == x.max()).nonzero()[0])
                onward = next((t for t in kids if tokens[first + t] == token), None)
            else:
                r, gone = p.exp(), 0.0
                for t in kids:
                    mine = tokens[first + t]
                    if inp["draft"] is None:
                        q = torch.zeros_like(r)
                        q[mine] = 1.0
                    else:
                        q = inp["draft"][first + at].double()
                        gone, q = gone + float(q[mine]), q / (1.0 - gone) if c["draft"] == "once" else q
                    if uniform[first + t] * float(q[mine]) < float(r[mine]):
                        onward = t
                        break
                    r = torch.relu(r - q)
                    r = r / r.sum()
                if onward is None:
                    token = int((torch.cumsum(r, 0) > uniform[first] * r.sum()).nonzero()[0])
            if onward is None:
                break
            log.append(float(p[tokens[first + onward]]))
            at = onward
        lengths.append(len(walk))
        path += walk + [-1] * (len(tree) - len(walk))
        following.append(token)
        logs += log + [float(p[token])] + [0.0] * (len(tree) - len(walk))
    return [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lengths, path, following)] + [torch.tensor(logs, dtype=torch.float64, device="cuda")]


def _exact_keep(c, inp, nodes, cached, chains):
    k, v = inp["k"].double(), inp["v"].double()
    for i, p in enumerate(cached):
        walk = [t for t in inp["paths"][i] if t >= 0]
        to = torch.arange(p, p + len(walk), device=k.device)
        at = torch.tensor([p + t for t in walk], device=k.device)
        for new, old in ((k, inp["k"]), (v, inp["v"])):
            _put(c, inp, new, i, to, _at(c, inp, old, i, at).double())
    ends = [p + sum(t >= 0 for t in w) for p, w in zip(cached, inp["paths"])]
    return [torch.tensor(ends, dtype=torch.int32, device=k.device), k, v]


EXACT = dict(append=_exact_append, attend=_exact_attend, verify=_exact_verify, keep=_exact_keep)
