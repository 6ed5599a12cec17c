"""What the tests of mpk_rows_* share: a small model's graph over a cache of torch tensors, and 64-bit results."""
import math
from types import SimpleNamespace

import torch

import paper_2512_22219_amd as M

BF16_HALF = torch.finfo(torch.bfloat16).eps / 2    # a rounding to bf16, relative to the value
F32_HALF = torch.finfo(torch.float32).eps / 2


class RowsModel:
    """A compiled graph of a tiny model with the wanted heads, its cache (bf16 [layers][slots or pages][kv][rows][d]) filled
    with `fill`, or normal values."""

    def __init__(self, n_q=4, n_kv=2, d=64, layers=2, batch=4, max_seq=192, page=0, pages=0, qk_norm=False, theta=1e4, vocab=64,
                 seed=0, fill=None, host_only=False, **opts):
        self.n_q, self.n_kv, self.d, self.batch, self.max_seq, self.page = n_q, n_kv, d, batch, max_seq, page
        self.theta, self.eps, self.vocab, self.layers, self.qk_norm = theta, 1e-6, vocab, layers, qk_norm
        self.shape = SimpleNamespace(n_layers=layers, hidden=64, n_q_heads=n_q, n_kv_heads=n_kv, head_dim=d, ffn=128, vocab=vocab,
                                     rms_eps=self.eps, rope_theta=theta, batch=batch, max_seq=max_seq, n_experts=0, top_k=0,
                                     expert_ffn=0, qk_norm=qk_norm)
        opts = dict(dict(fusion=31, transitive_reduction=1), **opts)
        if page:
            opts.update(kv_page_size=page, kv_pages=pages)
        if host_only:
            self.graph = M.compile_graph(self.shape, None, None, host_only=1, **opts)
            return
        dev = self.dev = torch.device("cuda")
        self.gen = torch.Generator(device=dev).manual_seed(seed)
        H, F, w = 64, 128, self.normal
        self.w = []
        for _ in range(layers):
            lw = dict(attn_norm=1 + w(H, std=0.02), wqkv=w((n_q + 2 * n_kv) * d, H, std=0.1), wo=w(H, n_q * d, std=0.1),
                      mlp_norm=1 + w(H, std=0.02), wgu=w(2 * F, H, std=0.1), wd=w(H, F, std=0.1))
            if qk_norm:
                lw.update(q_norm=1 + w(d, std=0.02), k_norm=1 + w(d, std=0.02))
            self.w.append(lw)
        self.outer = dict(embed=w(vocab, H), final_norm=1 + w(H, std=0.02), lm_head=w(vocab, H, std=0.1))
        size = (layers, pages if page else batch, n_kv, page or max_seq, d)
        self.k, self.v = (w(*size) if fill is None else torch.full(size, fill, dtype=torch.bfloat16, device=dev) for _ in range(2))
        ptrs = {n: t.data_ptr() for n, t in self.outer.items()}
        ptrs["layers"] = [{n: t.data_ptr() for n, t in lw.items()} for lw in self.w]
        self.graph = M.compile_graph(self.shape, ptrs, (self.k.data_ptr(), self.v.data_ptr()), **opts)
        if page:
            blocks = max_seq // page
            deal = torch.randperm(pages, generator=self.gen, device=dev)
            self.table = deal[torch.arange(batch * blocks, device=dev) % pages].view(batch, blocks).to(torch.int32)
            self.graph.set_page_table(self.table.data_ptr())

    def normal(self, *size, std=1.0, dtype=torch.bfloat16):
        return (torch.empty(size, dtype=torch.float32, device=self.dev).normal_(0, std, generator=self.gen)).to(dtype)

    def ints(self, values):
        return torch.tensor(values, dtype=torch.int32, device=self.dev)

    def cached(self, cache, layer, slot, n):
        """Rows 0 .. n - 1 of a slot: [kv][n][d]."""
        if not self.page:
            return cache[layer, slot, :, :n]
        pages = self.table[slot].long()
        return cache[layer][pages].transpose(0, 1).reshape(self.n_kv, -1, self.d)[:, :n]

    def append(self, layer, begin, slots, positions, qkv, q_out, n_rows=None, stream=None):
        kind = M.ROWS_F32 if qkv.dtype == torch.float32 else M.ROWS_BF16
        self.keep = (self.ints(begin), self.ints(slots) if slots is not None else None, self.ints(positions))
        b, s, p = self.keep
        self.graph.rows_append(layer, len(begin) - 1, qkv.shape[0] if n_rows is None else n_rows, b.data_ptr(),
                               s.data_ptr() if s is not None else 0, p.data_ptr(), qkv.data_ptr(), kind, qkv.stride(0),
                               q_out.data_ptr(), q_out.stride(0), _stream(stream))

    def attend(self, layer, begin, slots, positions, q, out, work, n_rows=None, stream=None):
        self.keep = (self.ints(begin), self.ints(slots) if slots is not None else None, self.ints(positions))
        b, s, p = self.keep
        self.graph.rows_attend(layer, len(begin) - 1, q.shape[0] if n_rows is None else n_rows, b.data_ptr(),
                               s.data_ptr() if s is not None else 0, p.data_ptr(), q.data_ptr(), q.stride(0), out.data_ptr(),
                               out.stride(0), work.data_ptr(), _stream(stream))

    def status(self):
        torch.cuda.synchronize()
        self.graph.status()


def _stream(stream):
    return torch.cuda.current_stream().cuda_stream if stream is None else stream


def workspace():
    """Filled with NaN patterns: what a call reads there it has written."""
    return torch.full((M.ROWS_WORKSPACE_BYTES // 4,), float("nan"), dtype=torch.float32, device="cuda")


def append_exact(m, layer, pos, x):
    """x [rows][heads * d] at positions pos [rows] -> q, k, v in 64 bits [rows][heads][d] and the size of what the rotation adds."""
    x = x.double().view(len(pos), -1, m.d)
    q, k, v = x.split((m.n_q, m.n_kv, m.n_kv), 1)
    if m.qk_norm:
        q, k = (y / torch.sqrt(y.square().mean(-1, keepdim=True) + m.eps) * m.w[layer][g].double()
                for y, g in ((q, "q_norm"), (k, "k_norm")))
    f = m.theta ** (-2.0 * torch.arange(m.d // 2, dtype=torch.float64, device=x.device) / m.d)
    a = (pos.double()[:, None] * f)[:, None]
    out = []
    for y in (q, k):
        lo, hi = y[..., : m.d // 2], y[..., m.d // 2:]
        size = (lo.abs() + hi.abs()).repeat(1, 1, 2)
        out += [torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1), size]
    return out[0], out[2], v, out[1], out[3]


def attend_exact(q, k, v, pos):
    """q [rows][n_q][d], k and v [kv][n][d], pos [rows] -> the output in 64 bits, and a bound on the error of a kernel that
    keeps scores and sums in 32 bits, rounds the probabilities to bf16 for the product with V and the output once."""
    q, k, v = q.double(), k.double(), v.double()
    rows, n_q, d = q.shape
    q = q.view(rows, k.shape[0], -1, d).transpose(0, 1)                                   # [kv][rows][g][d]
    kt, n = k[:, None].transpose(2, 3), k.shape[1]
    seen = (torch.arange(n, device=q.device)[None, :] <= pos[:, None])[None, :, None]      # [1][rows][1][n]
    s = (q @ kt).masked_fill(~seen, -math.inf) / math.sqrt(d)
    w = torch.softmax(s, -1)
    o, mean_abs = w @ v[:, None], w @ v[:, None].abs()
    # a score: d products and additions in 32 bits, the scale, the distance to the maximum, the exponential (two steps)
    size = ((q.abs() @ kt.abs()).masked_fill(~seen, 0.0) / math.sqrt(d)).amax(-1, keepdim=True)
    delta = 2 * (d + 8) * F32_HALF * size + 8 * F32_HALF
    # sums of n weights, merged from parts
    delta = delta + (n / 16 + 64) * F32_HALF
    bound = BF16_HALF * o.abs() + (BF16_HALF + 2 * delta) * mean_abs * (1 + BF16_HALF)
    back = lambda y: y.transpose(0, 1).reshape(rows, n_q, d)  # noqa: E731
    return back(o), back(bound)
