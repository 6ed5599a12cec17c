"""Rows beside the decode step, measured: filling a graph's KV cache with many rows at once
(`Graph.rows_append`), attention of those rows over the cache (`Graph.rows_attend`), and what rows of
logits say about tokens (`Graph.rows_logprobs`).

A case is one call of one of them, for one layer: a serving program makes the first two once a layer for
every chunk of prompts, the third once a step or once a scored prompt.  With `own` false the same results
come from elementary torch operations in 32 bits (angles in 64).

Queries, keys and values are N(0, 1), gains 1 + N(0, 0.02), as in the repository's synthetic models;
logits are N(0, 2.5) with one token a row raised by 0 .. 15, so that rows are anything from flat to certain.
"""
import math
import random
from types import SimpleNamespace

import torch

import paper_2512_22219_amd as M

own = False
EPS = 1e-6


def _rows(name, op, **kw):
    # new, cached: rows of a sequence in the call, and before it, from .. to over the sequences
    c = dict(op=op, q_heads=32, kv_heads=8, head_dim=128, theta=1e6, qk_norm=False, seqs=1, new_lo=1, new_hi=1,
             cached_lo=0, cached_hi=0, page=0, type="bf16")
    c.update(kw)
    if name:
        c["name"] = name
    return c


def _logits(name, **kw):
    c = dict(op="logprobs", rows=1, vocab=151936, top=20, type="f32", masked=False)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest call: one new token of one request, the 8B shape with the query/key norm; nothing but latency
        _rows("append 1 token", "append", qk_norm=True, cached_lo=1024, cached_hi=1024),
        # eight requests' prompts of a mixed length in one call, fp32 projections, pages of 16 rows: what admission of a
        # burst looks like on the serving cache
        _rows("append 8 ragged prompts, paged", "append", theta=5e5, seqs=8, new_lo=17, new_hi=500, cached_lo=0,
              cached_hi=3000, page=16, type="f32"),
        # a long prompt's chunk on the 70B shape, eight query heads per KV head
        _rows("append 8192 tokens", "append", q_heads=64, theta=5e5, new_lo=8192, new_hi=8192),
        # one token of eight requests with the benchmark's ragged cache lengths: the single-token form, all memory
        _rows("attend 8 x 1 token", "attend", theta=5e5, seqs=8, cached_lo=512, cached_hi=4096),
        # a few drafted tokens checked against one long cache, head size 64, pages of 16: split over the long axis
        _rows("attend 5 tokens over 30000, paged", "attend", head_dim=64, new_lo=5, new_hi=5, cached_lo=30001,
              cached_hi=30001, page=16),
        # the offline workload's prompt of 64 tokens, no cache before it: a short call
        _rows("attend 64 tokens", "attend", new_lo=64, new_hi=64),
        # sixteen requests in one call, some with a prompt, some with a single token, four KV heads, pages of 64
        _rows("attend 16 ragged, paged", "attend", kv_heads=4, seqs=16, new_lo=1, new_hi=700, cached_lo=0,
              cached_hi=2100, page=64),
        # a whole prompt of 4096 tokens at once
        _rows("attend 4096 tokens", "attend", theta=5e5, new_lo=4096, new_hi=4096),
        # the largest: a chunk of 2048 tokens behind 14000 cached ones on the 70B shape
        _rows("attend 2048 tokens over 14000", "attend", q_heads=64, theta=5e5, new_lo=2048, new_hi=2048,
              cached_lo=14000, cached_hi=14000),
        # one token of one request with twenty alternatives: the smallest scoring call
        _logits("logprobs 1 row"),
        # a step of sixteen requests under a grammar that rules most tokens out
        _logits("logprobs 16 rows, masked", rows=16, vocab=128256, top=5, masked=True),
        # a prompt of 4096 tokens scored, logits in bf16 as a matrix product leaves them
        _logits("logprobs 4096 rows", rows=4096, vocab=32000, top=4, type="bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "logprobs"])
    if op == "logprobs":
        c = _logits(None, vocab=_log(rng, 1000, 152000), top=rng.choice([0, 1, 4, 5, 20, 32]), type=rng.choice(["f32", "bf16"]),
                    masked=rng.random() < 0.25)
        c["rows"] = _log(rng, 1, max(2, min(8192, (1 << 27) // c["vocab"])))
        return c
    c = _rows(None, op, head_dim=rng.choice([64, 128]), theta=rng.choice([1e4, 5e5, 1e6]), qk_norm=rng.random() < 0.5,
              seqs=rng.choice([1, 1, 2, 3, 5, 8, 13, 16]), page=rng.choice([0, 0, 8, 16, 64]), type=rng.choice(["bf16", "f32"]))
    c["kv_heads"] = rng.choice([2, 4, 8])
    c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 8])
    c["new_hi"] = _log(rng, 1, 8192 // c["seqs"])
    c["new_lo"] = rng.choice([1, c["new_hi"], rng.randint(1, c["new_hi"])])
    c["cached_hi"] = _log(rng, 1, 32000 // c["seqs"]) - 1
    c["cached_lo"] = rng.choice([0, c["cached_hi"], rng.randint(0, c["cached_hi"])])
    if op == "attend":
        c["type"] = "bf16"
        while c["seqs"] * c["q_heads"] * c["new_hi"] * (c["cached_hi"] + c["new_hi"]) > 1 << 31:   # (the plain form's scores)
            if c["new_hi"] > c["cached_hi"]:
                c["new_hi"] = c["new_hi"] // 2 + 1
                c["new_lo"] = min(c["new_lo"], c["new_hi"])
            else:
                c["cached_hi"] = c["cached_hi"] // 2
                c["cached_lo"] = min(c["cached_lo"], c["cached_hi"])
    return c


def _lens(c):
    """(new rows, rows cached before) of every sequence: spread over their ranges, in a mixed order, the largest first."""
    n = c["seqs"]

    def spread(lo, hi, step):
        return [hi - (hi - lo) * (i * step % n) // max(1, n - 1) for i in range(n)]

    odd = next(s for s in (5, 7, 11) if n % s)
    return spread(c["new_lo"], c["new_hi"], 1), spread(c["cached_lo"], c["cached_hi"], odd)


# ---------------------------------------------------------------------------------- inputs
def _inputs(c, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*size, std=1.0, dtype=torch.bfloat16):
        return torch.empty(size, dtype=dtype, device=dev).normal_(0.0, std, generator=gen)

    dtype = torch.float32 if c["type"] == "f32" else torch.bfloat16
    if c["op"] == "logprobs":
        x = normal(c["rows"], c["vocab"], std=2.5, dtype=torch.float32)
        top = torch.randint(c["vocab"], (c["rows"],), generator=gen, device=dev)
        other = torch.randint(c["vocab"], (c["rows"],), generator=gen, device=dev)
        if c["masked"]:   # what a grammar rules out is at -inf; the tokens asked for are not
            out = torch.rand(c["rows"], c["vocab"], generator=gen, device=dev) < 0.9
            out.scatter_(1, torch.stack([top, other], 1), False)
            x.masked_fill_(out, -math.inf)
        x.scatter_add_(1, top[:, None], 15 * torch.rand(c["rows"], 1, generator=gen, device=dev))
        pick = torch.rand(c["rows"], generator=gen, device=dev) < 0.5
        return {"logits": x.to(dtype), "tokens": torch.where(pick, top, other).to(torch.int32)}
    new, cached = _lens(c)
    nkv, d, n = c["kv_heads"], c["head_dim"], c["seqs"]
    rows, step = sum(new), c["page"] or 8
    max_seq = -(-max(a + b for a, b in zip(new, cached)) // step) * step
    inp = {"max_seq": max_seq, "rows": rows, "longest": max(new), "pages": 0}
    begin = [sum(new[:i]) for i in range(n + 1)]
    inp["row_begin"] = torch.tensor(begin, dtype=torch.int32, device=dev)
    inp["positions"] = torch.tensor(cached, dtype=torch.int32, device=dev)
    if c["page"]:   # every sequence's blocks in pages of a shuffled pool
        blocks = max_seq // c["page"]
        inp["pages"] = n * blocks + 3
        deal = torch.randperm(inp["pages"], generator=gen, device=dev)
        inp["table"] = deal[: n * blocks].view(n, blocks).to(torch.int32)
        size = (1, inp["pages"], nkv, c["page"], d)
    else:
        size = (1, n, nkv, max_seq, d)
    inp["k"], inp["v"] = normal(*size), normal(*size)
    heads = c["q_heads"] + (2 * nkv if c["op"] == "append" else 0)
    inp["x"] = normal(rows, heads * d, dtype=dtype)
    for g in ("q_norm", "k_norm"):
        inp[g] = (1.0 + normal(d, std=0.02, dtype=torch.float32)).to(torch.bfloat16)
    inp["inv_freq"] = c["theta"] ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=dev) / d)
    return inp


def _graph(c, inp):
    """The compiled graph that the calls belong to: one small layer of the case's heads, over the case's cache."""
    dev, bf = torch.device("cuda"), torch.bfloat16
    scoring = c["op"] == "logprobs"
    nq, nkv, d = (4, 2, 64) if scoring else (c["q_heads"], c["kv_heads"], c["head_dim"])
    H, F, V = 128, 256, c["vocab"] if scoring else 1024
    batch, max_seq = (1, 64) if scoring else (c["seqs"], inp["max_seq"])
    norm = not scoring and c["qk_norm"]
    shape = SimpleNamespace(n_layers=1, hidden=H, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, ffn=F, vocab=V, rms_eps=EPS,
                            rope_theta=1e4 if scoring else c["theta"], batch=batch, max_seq=max_seq, n_experts=0, top_k=0,
                            expert_ffn=0, qk_norm=norm)

    def zeros(*size):
        return torch.zeros(size, dtype=bf, device=dev)

    w = {"attn_norm": zeros(H), "wqkv": zeros((nq + 2 * nkv) * d, H), "wo": zeros(H, nq * d), "mlp_norm": zeros(H),
         "wgu": zeros(2 * F, H), "wd": zeros(H, F)}
    if norm:
        w.update(q_norm=inp["q_norm"], k_norm=inp["k_norm"])
    outer = {"embed": zeros(V, H), "final_norm": zeros(H), "lm_head": zeros(V, H)}
    k, v = (zeros(1, 1, nkv, max_seq, d), zeros(1, 1, nkv, max_seq, d)) if scoring else (inp["k"], inp["v"])
    ptrs = {n: t.data_ptr() for n, t in outer.items()}
    ptrs["layers"] = [{n: t.data_ptr() for n, t in w.items()}]
    paged = {} if scoring or not c["page"] else dict(kv_page_size=c["page"], kv_pages=inp["pages"])
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
    if c["op"] == "logprobs":
        R, k = c["rows"], c["top"]
        st["logprobs"] = torch.empty(R, dtype=torch.float32, device=dev)
        st["entropy"] = torch.empty(R, dtype=torch.float32, device=dev)
        st["top_tokens"] = torch.empty((R, k), dtype=torch.int32, device=dev)
        st["top_logprobs"] = torch.empty((R, k), dtype=torch.float32, device=dev)
    else:
        st["out"] = torch.empty((inp["rows"], c["q_heads"] * c["head_dim"]), dtype=torch.bfloat16, device=dev)
    torch.cuda.synchronize()
    return st


# ---------------------------------------------------------------------------------- one pass
def run(st):
    c, inp = st["case"], st["inputs"]
    if c["op"] == "logprobs":
        return _own_logprobs(st) if own else _plain_logprobs(c, inp)
    if c["op"] == "append":
        return _own_append(st) if own else _plain_append(c, inp)
    return _own_attend(st) if own else _plain_attend(c, inp)


def _own_append(st):
    c, inp, g = st["case"], st["inputs"], st["graph"]
    g.rows_append(0, c["seqs"], inp["rows"], inp["row_begin"].data_ptr(), 0, inp["positions"].data_ptr(), inp["x"].data_ptr(),
                  M.ROWS_F32 if c["type"] == "f32" else M.ROWS_BF16, inp["x"].stride(0), st["out"].data_ptr(),
                  st["out"].stride(0), torch.cuda.current_stream().cuda_stream)
    return [st["out"], inp["k"], inp["v"]]


def _own_attend(st):
    c, inp, g = st["case"], st["inputs"], st["graph"]
    g.rows_attend(0, c["seqs"], inp["rows"], inp["row_begin"].data_ptr(), 0, inp["positions"].data_ptr(), inp["x"].data_ptr(),
                  inp["x"].stride(0), st["out"].data_ptr(), st["out"].stride(0), st["work"].data_ptr(),
                  torch.cuda.current_stream().cuda_stream)
    return [st["out"]]


def _own_logprobs(st):
    c, inp, g = st["case"], st["inputs"], st["graph"]
    x = inp["logits"]
    g.rows_logprobs(c["rows"], x.data_ptr(), M.ROWS_F32 if c["type"] == "f32" else M.ROWS_BF16, x.stride(0),
                    inp["tokens"].data_ptr(), c["top"], st["logprobs"].data_ptr(), st["entropy"].data_ptr(),
                    st["top_tokens"].data_ptr(), st["top_logprobs"].data_ptr(), st["work"].data_ptr(),
                    torch.cuda.current_stream().cuda_stream)
    return [st["logprobs"], st["entropy"], st["top_tokens"], st["top_logprobs"]]


def _row_places(inp):
    """The sequence of every row, its place in the sequence and its position."""
    r = torch.arange(inp["rows"], device=inp["row_begin"].device)
    seq = (r[:, None] >= inp["row_begin"][None, 1:]).sum(1)
    t = r - inp["row_begin"][seq]
    return seq, t, t + inp["positions"][seq]


def _plain_append(c, inp):
    nq, nkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    x = inp["x"].float().view(inp["rows"], nq + 2 * nkv, d)
    q, k, v = x.split((nq, nkv, nkv), 1)
    if c["qk_norm"]:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + EPS) * inp["q_norm"].float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + EPS) * inp["k_norm"].float()
    seq, _, pos = _row_places(inp)
    angle = pos.double()[:, None] * inp["inv_freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = torch.cat([q, k], 1)
    lo, hi = x[..., : d // 2], x[..., d // 2:]
    x = torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).to(torch.bfloat16)
    if c["page"]:
        at, row = inp["table"][seq, pos // c["page"]].long(), pos % c["page"]
    else:
        at, row = seq, pos
    inp["k"][0][at, :, row] = x[:, nq:]
    inp["v"][0][at, :, row] = v.to(torch.bfloat16)
    return [x[:, :nq].reshape(inp["rows"], nq * d), inp["k"], inp["v"]]


def _plain_attend(c, inp):
    nq, nkv, d, n = c["q_heads"], c["kv_heads"], c["head_dim"], c["seqs"]
    G, T, S = nq // nkv, inp["longest"], inp["max_seq"]
    k, v = inp["k"][0], inp["v"][0]
    if c["page"]:
        k, v = (x[inp["table"].long()].transpose(1, 2).reshape(n, nkv, S, d) for x in (k, v))
    t = torch.arange(T, device=k.device)
    rows = (inp["row_begin"][:-1, None] + t).clamp(max=inp["rows"] - 1)
    q = inp["x"].float()[rows].view(n, T, nkv, G, d).permute(0, 2, 3, 1, 4).reshape(n, nkv, G * T, d)
    s = torch.matmul(q, k.float().transpose(2, 3)).view(n, nkv, G, T, S)
    seen = torch.arange(S, device=k.device) <= (inp["positions"][:, None] + t)[..., None]
    s = (s * d ** -0.5).masked_fill_(~seen[:, None, None], -math.inf)
    s = (s - s.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(s.view(n, nkv, G * T, S), v.float()).view(n, nkv, G, T, d) / s.sum(-1, keepdim=True)
    seq, t, _ = _row_places(inp)
    return [o.permute(0, 3, 1, 2, 4)[seq, t].reshape(inp["rows"], nq * d).to(torch.bfloat16)]


def _plain_logprobs(c, inp):
    x = inp["logits"].float()
    below = x - x.amax(1, keepdim=True)
    e = below.exp()
    total = e.sum(1)
    norm = total.log()
    entropy = norm - torch.where(e > 0, e * below, 0.0).sum(1) / total
    given = below.gather(1, inp["tokens"].long()[:, None])[:, 0] - norm
    # the largest logits, of equal ones the lowest index first: one whole number of both, so that nothing ties
    bits = (x + 0.0).view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + (0x7FFFFFFF - torch.arange(c["vocab"], device=x.device))
    tokens = 0x7FFFFFFF - (order.topk(c["top"], 1).values & 0xFFFFFFFF)
    return [given, entropy, tokens.to(torch.int32), below.gather(1, tokens) - norm[:, None]]


# ---------------------------------------------------------------------------------- what a pass needs
def work(case):
    c = case
    size = 4 if c["type"] == "f32" else 2
    if c["op"] == "logprobs":
        values = c["rows"] * c["vocab"]
        return {"bytes": float(values * size + c["rows"] * (12 + 8 * c["top"])), "flops": 6.0 * values}
    new, cached = _lens(c)
    nq, nkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    if c["op"] == "append":
        values = sum(new) * (nq + 2 * nkv) * d
        return {"bytes": float(values * (size + 2)), "flops": 10.0 * values}
    pairs = sum(t * p + t * (t + 1) // 2 for t, p in zip(new, cached))
    return {"bytes": 4.0 * (sum(new) * nq * d + sum(t + p for t, p in zip(new, cached)) * nkv * d), "flops": 4.0 * pairs * nq * d}


# ---------------------------------------------------------------------------------- 64-bit results
def exact(case, seed):
    c, inp = case, _inputs(case, seed)
    if c["op"] == "logprobs":
        outs = [[], [], []]
        for x, tok in zip(inp["logits"].split(256), inp["tokens"].split(256)):
            p = torch.log_softmax(x.double(), -1)
            outs[0].append(p[torch.arange(len(tok)), tok.long()])
            outs[1].append(-(p.exp() * p.clamp(min=-1e4)).sum(-1))
            outs[2].append(p.sort(-1, descending=True).values[:, : c["top"]])
        given, entropy, best = (torch.cat(o) for o in outs)
        return [given, entropy, None, best]
    new, cached = _lens(c)
    nq, nkv, d, P = c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    k, v = inp["k"][0].double(), inp["v"][0].double()
    out, first = [], 0
    if c["op"] == "append":
        for i, (T, p) in enumerate(zip(new, cached)):
            x = inp["x"][first:first + T].double().view(T, nq + 2 * nkv, d)
            at = torch.arange(p, p + T, device=x.device)
            q, kk, vv = x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:]
            if c["qk_norm"]:
                q, kk = (y / torch.sqrt((y * y).sum(-1, keepdim=True) / d + EPS) * inp[g].double()
                         for y, g in ((q, "q_norm"), (kk, "k_norm")))
            turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), at.double()[:, None] * inp["inv_freq"])[:, None]
            q, kk = (torch.cat([z.real, z.imag], -1) for z in (torch.complex(y[..., : d // 2].contiguous(), y[..., d // 2:].contiguous()) * turn
                                                               for y in (q, kk)))
            out.append(q.reshape(T, nq * d))
            if P:
                pg = inp["table"][i].long()[at // P]
                k[pg, :, at % P], v[pg, :, at % P] = kk, vv
            else:
                k[i, :, p:p + T], v[i, :, p:p + T] = kk.transpose(0, 1), vv.transpose(0, 1)
            first += T
        return [torch.cat(out), k[None], v[None]]
    for i, (T, p) in enumerate(zip(new, cached)):
        q = inp["x"][first:first + T].double().view(T, nkv, nq // nkv, d)
        hidden = torch.arange(p + T, device=q.device)[None, :] > torch.arange(p, p + T, device=q.device)[:, None]
        o = torch.empty_like(q)
        for h in range(nkv):
            kh, vh = (x[inp["table"][i].long(), h].reshape(-1, d)[: p + T] if P else x[i, h, : p + T] for x in (k, v))
            for g in range(nq // nkv):
                s = (q[:, h, g] @ kh.t() / math.sqrt(d)).masked_fill(hidden, -math.inf)
                o[:, h, g] = torch.softmax(s, -1) @ vh
        out.append(o.reshape(T, nq * d))
        first += T
    return [torch.cat(out)]
