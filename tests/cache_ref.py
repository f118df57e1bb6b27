"""The operators of the uncompressed cache in float64 on the CPU, written from their definitions, and the bounds on what
a kernel's float32 sums and roundings to the storage type may put between its result and these.  Test infrastructure."""
import math

import torch

D = 128
U32 = 2.0 ** -24                     # half a step of float32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def spans(B, n_rows, q_start):
    """Per sequence: first row and number of its new tokens."""
    if q_start is None:
        return [(b, 1) for b in range(B)]
    out = []
    for b in range(B):
        lo = min(max(int(q_start[b]), 0), n_rows)
        out.append((lo, min(max(int(q_start[b + 1]), lo), n_rows) - lo))
    return out


def token_row(pool, table, b, j):
    """The page and the row of token j of sequence b, or None."""
    ps = pool.shape[2]
    page = b if table is None else int(table[b, j // ps])
    return (page, j % ps) if 0 <= page < pool.shape[0] else None


def capacity(pool, table):
    return pool.shape[2] * (1 if table is None else table.shape[1])


def rotate(x, w, pos, inv_freq, eps, pairs):
    """x [n, heads, D] float64 at positions pos -> (result, |x| + |partner|: what the rounding errors are relative to)."""
    y = x.double()
    if w is not None:
        y = y / (y.pow(2).mean(-1, keepdim=True) + eps).sqrt() * w.double()
    size = y.abs()
    n = 0 if inv_freq is None else inv_freq.numel()
    if n:
        a = torch.outer(pos.double(), inv_freq)[:, None]
        i = torch.arange(n)
        lo, hi = (2 * i, 2 * i + 1) if pairs else (i, i + n)
        u, v = y[..., lo], y[..., hi]
        y = y.clone()
        y[..., lo], y[..., hi] = u * a.cos() - v * a.sin(), v * a.cos() + u * a.sin()
        size = size.clone()
        size[..., lo] = size[..., hi] = u.abs() + v.abs()
    return y, size


def rotate_bound(ref, size, dtype):
    """Half a step of the storage type, and 32 half steps of float32 for the sum of 128 squares (a tree behind 8 in a row),
    root, three products, cosine and sine (3 steps each) and the last sum."""
    return half_step(dtype) * ref.abs() * 1.01 + 32 * U32 * size


def attend(q, pool_k, pool_v, table, n_ctx, q_start, scale, window, n_sink, n_cap, Hkv):
    """-> dict of out [n_rows, Hq, D], rows (which rows are somebody's), weight = sum p |v|, scores [B, Hkv, n_cap] (the
    growth), e (largest error of a logit) and seen [n_rows]."""
    n_rows, Hq, _ = q.shape
    B, G, cap = len(n_ctx), q.shape[1] // Hkv, capacity(pool_k, table)
    out = torch.zeros(n_rows, Hq, D, dtype=torch.float64)
    weight = torch.zeros_like(out)
    scores = torch.zeros(B, Hkv, n_cap, dtype=torch.float64)
    rows = torch.zeros(n_rows, dtype=torch.bool)
    e = 0.0
    for b, (r0, y) in enumerate(spans(B, n_rows, q_start)):
        rows[r0:r0 + y] = True
        n = min(max(int(n_ctx[b]), 0), cap)
        at = [(j, token_row(pool_k, table, b, j)) for j in range(n)]
        at = [(j, pr) for j, pr in at if pr is not None]
        if not at or y == 0:
            continue
        j = torch.tensor([x for x, _ in at])
        page, row = torch.tensor([pr[0] for _, pr in at]), torch.tensor([pr[1] for _, pr in at])
        P = torch.arange(n - y, n)[:, None]
        seen = (j <= P) & ((j > P - window) | (j < n_sink) if window else True)
        used = seen.any(0)                                  # tokens that no query sees may hold anything
        j, page, row, seen = j[used], page[used], row[used], seen[:, used]
        if j.numel() == 0:
            continue
        keep = j < n_cap
        for h in range(Hkv):
            k, v = pool_k[page, h, row].double(), pool_v[page, h, row].double()
            for g in range(G):
                x = q[r0:r0 + y, h * G + g].double()
                s = x @ k.T * scale
                # 130 roundings of a sum of 128 products, relative to the sum of their sizes
                e = max(e, float((x.abs() @ k.abs().T)[seen].max() if seen.any() else 0) * abs(scale) * 130 * U32)
                s = s.masked_fill(~seen, -math.inf)
                p = (s - s.amax(-1, keepdim=True).clamp(min=-1e300)).exp()
                total = p.sum(-1, keepdim=True)
                p = torch.where(total > 0, p / total.clamp(min=1e-300), torch.zeros_like(p))
                # a token that this query does not see does not count, whatever it holds
                out[r0:r0 + y, h * G + g] = p @ torch.where(torch.isfinite(v), v, torch.zeros_like(v))
                bad = (~torch.isfinite(v)).any(-1)
                for i in bad.nonzero()[:, 0].tolist():
                    t = seen[:, i].nonzero()[:, 0]
                    z = torch.where(torch.isfinite(v[i]), torch.zeros_like(v[i]), v[i])
                    out[r0 + t, h * G + g] += p[t, i][:, None] * z
                weight[r0:r0 + y, h * G + g] = p @ torch.nan_to_num(v.abs(), posinf=0.0)
                scores[b, h].index_add_(0, j[keep], p.sum(0)[keep])
    return dict(out=out, weight=weight, scores=scores, rows=rows, e=e)


def attend_bounds(ref, dtype, old_scores=None):
    """Bounds on |out - ref| and |scores - ref|.  A weight p = exp(s - m) / sum is off by the error of its logit, by the
    roundings of s - m and of its exponential (|s - m| < 100 where it counts: 2^-16) and as much again through the sum;
    where the storage type is bf16 also by rounding it to bf16 for the product with the values.  The output is rounded
    to the storage type; sums of n weights in float32 tiles: 2^-14 covers n = 1024 roundings."""
    rel = 2 * (ref["e"] + 2.0 ** -16) + 2.0 ** -14
    u = half_step(dtype)
    low = u if dtype == torch.bfloat16 else 0.0
    out = u * ref["out"].abs() + (rel + low) * 1.01 * ref["weight"] + 1e-30
    sc = rel * ref["scores"] + 1e-30
    if old_scores is not None:
        sc = sc + 4 * U32 * (old_scores.double().abs() + ref["scores"])
    return out, sc
