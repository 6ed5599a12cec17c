"""What the tests of mpk_tree_* share: trees, the calls on a small model's graph, and 64-bit results."""
import math
import random

import torch

import paper_2512_22219_amd as M
from tests.rows_util import BF16_HALF, F32_HALF, RowsModel, _stream, workspace


def tree(nodes, kind="random", seed=0, roots=1):
    """Parents: a chain, a star, two branches, or at random (several roots for more trees than one)."""
    rng = random.Random(seed)
    out = []
    for t in range(nodes):
        if t < roots:
            out.append(-1)
        elif kind == "chain":
            out.append(t - 1)
        elif kind == "star":
            out.append(t % roots)
        elif kind == "two":   # nodes in turn: no node's parent is the one in front of it
            out.append(max(0, t - 2))
        else:
            out.append(rng.randrange(max(0, t - 12), t))
    return out


def chains(parents):
    """Per node: its ancestors, the first first, and itself."""
    out = []
    for t, p in enumerate(parents):
        out.append((out[p] if p >= 0 else []) + [t])
    return out


class TreeModel(RowsModel):
    def _lists(self, begin, slots, positions, *more):
        self.keep_alive = [self.ints(x) if x is not None else None for x in (begin, slots, positions, *more)]
        return [x.data_ptr() if x is not None else 0 for x in self.keep_alive]

    def tree_append(self, layer, begin, slots, positions, parents, qkv, q_out, n_rows=None, stream=None):
        b, s, p, t = self._lists(begin, slots, positions, parents)
        kind = M.ROWS_F32 if qkv.dtype == torch.float32 else M.ROWS_BF16
        self.graph.tree_append(layer, len(begin) - 1, qkv.shape[0] if n_rows is None else n_rows, b, s, p, t, qkv.data_ptr(), kind,
                               qkv.stride(0), q_out.data_ptr(), q_out.stride(0), _stream(stream))

    def tree_attend(self, layer, begin, slots, positions, parents, q, out, work, n_rows=None, stream=None):
        b, s, p, t = self._lists(begin, slots, positions, parents)
        self.graph.tree_attend(layer, len(begin) - 1, q.shape[0] if n_rows is None else n_rows, b, s, p, t, q.data_ptr(), q.stride(0),
                               out.data_ptr(), out.stride(0), work.data_ptr(), _stream(stream))

    def verify(self, begin, parents, tokens, logits, work, draft=None, once=False, temperatures=None, uniforms=None, n_rows=None,
               logprobs=True, stream=None, out=None):
        """lengths, path, next tokens, logprobs (all rows; of nobody's and where nothing is written 77)."""
        rows = len(parents) if n_rows is None else n_rows
        n = len(begin) - 1
        dev = logits.device
        if out is None:
            out = [torch.full((k,), 77, dtype=torch.int32, device=dev) for k in (n, max(1, rows), n)] + [torch.full((max(1, rows),), 77.0, device=dev)]
        lists = [torch.tensor(x, dtype=torch.int32, device=dev) for x in (begin, parents, tokens)]
        floats = [None if x is None else torch.as_tensor(x, dtype=torch.float32, device=dev) for x in (temperatures, uniforms)]
        self.keep_alive = lists + floats
        at = lambda x: 0 if x is None else x.data_ptr()  # noqa: E731
        self.graph.tree_verify(n, rows, *map(at, lists), at(logits), M.ROWS_F32 if logits.dtype == torch.float32 else M.ROWS_BF16,
                               logits.stride(0), at(draft), draft.stride(0) if draft is not None else 0, M.TREE_DRAWN_ONCE if once else 0,
                               *map(at, floats), *map(at, out[:3]), at(out[3]) if logprobs else 0, at(work), _stream(stream))
        return out

    def keep(self, begin, slots, positions, lengths, path, out=None, n_rows=None, stream=None):
        b, s, p, n, w = self._lists(begin, slots, positions, lengths, path)
        self.graph.tree_keep(len(begin) - 1, len(path) if n_rows is None else n_rows, b, s, p, n, w, 0 if out is None else out.data_ptr(),
                             _stream(stream))


def tree_attend_exact(q, k, v, pos, parents):
    """q [nodes][n_q][d], k and v [kv][pos + nodes][d] -> the output in 64 bits and a bound on the error of a kernel that keeps scores
    and sums in 32 bits, rounds the probabilities to bf16 for the product with V and the output once."""
    nodes, n_q, d = q.shape
    n = pos + nodes
    seen = torch.zeros(nodes, n, dtype=torch.bool)
    seen[:, :pos] = True
    for t, chain in enumerate(chains(parents)):
        seen[t, [pos + a for a in chain]] = True
    seen = seen.to(q.device)[None, :, None]
    # what no node sees may hold anything
    hidden = ~seen.any(1).view(1, n, 1)
    q, k, v = q.double(), k.double().masked_fill(hidden, 0.0), v.double().masked_fill(hidden, 0.0)
    q = q.view(nodes, k.shape[0], -1, d).transpose(0, 1)
    kt = k[:, None].transpose(2, 3).contiguous()
    s = (q @ kt).masked_fill(~seen, -math.inf) / math.sqrt(d)
    w = torch.softmax(s, -1)
    o, mean_abs = w @ v[:, None], w @ v[:, None].abs()
    # a score: d products and additions in 32 bits, the scale, the distance to the maximum, the exponential (two steps)
    size = ((q.abs() @ kt.abs()).masked_fill(~seen, 0.0) / math.sqrt(d)).amax(-1, keepdim=True)
    delta = 2 * (d + 8) * F32_HALF * size + 8 * F32_HALF
    delta = delta + (n / 16 + 64) * F32_HALF   # sums of n weights, merged from parts
    bound = BF16_HALF * o.abs() + (BF16_HALF + 2 * delta) * mean_abs * (1 + BF16_HALF)
    back = lambda y: y.transpose(0, 1).reshape(nodes, n_q, d)  # noqa: E731
    return back(o), back(bound)


def verify_exact(parents, tokens, logits, temperature, uniforms, draft=None, once=False):
    """One tree by the definition, in 64 bits on the CPU: path, next token, logprobs of the path."""
    at, path, logs = 0, [], []
    temperature = float(torch.tensor(temperature, dtype=torch.float32))   # (what the call is given)
    vocab = logits.shape[1]
    while True:
        path.append(at)
        x = logits[at].double().cpu()
        if not (x.max() < math.inf) or not (x.max() > -math.inf) or torch.isnan(x).any():
            return path, -1, logs + [math.nan]
        p = torch.log_softmax(x / (temperature or 1.0), 0)
        r, gone, onward = p.exp(), 0.0, None
        first = int((x == x.max()).nonzero()[0])
        for t in [t for t, q in enumerate(parents) if q == at and t > at]:
            mine = tokens[t]
            if not 0 <= mine < vocab:
                continue
            if temperature == 0:
                if mine == first:
                    onward = t
                    break
                continue
            if draft is None:
                q = torch.zeros(vocab, dtype=torch.float64)
                q[mine] = 1.0
            else:
                if once and gone >= 1.0:
                    continue
                q = draft[at].double().cpu()
                gone, q = gone + float(q[mine]), q / (1.0 - gone) if once else q
            if float(uniforms[t]) * float(q[mine]) < float(r[mine]):
                onward = t
                break
            rest = torch.relu(r - q)
            if rest.sum() > 0:
                r = rest / rest.sum()
        if onward is None:
            if temperature == 0:
                token = first
            else:
                below = torch.cumsum(r, 0)
                token = int((below > float(uniforms[0]) * float(below[-1])).nonzero()[0])
            return path, token, logs + [float(p[token])]
        logs.append(float(p[tokens[onward]]))
        at = onward


__all__ = ["BF16_HALF", "F32_HALF", "TreeModel", "chains", "tree", "tree_attend_exact", "verify_exact", "workspace"]
