"""The operators of a decoding step in 64 bits, with bounds on what fp32 arithmetic may add, element by element."""
import math

import numpy as np
import torch

import paper_2305_14405_b200 as nm

U = 2.0 ** -24                                     # half a step of fp32, relative
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}
RANGES = {"gelu": (nm.SLOT_GELU, nm.FUNC_GELU, 64, -4.0, 4.0), "exp": (nm.SLOT_EXP, nm.FUNC_EXP, 256, -16.0, 0.0),
          "recip": (nm.SLOT_RECIP, nm.FUNC_RECIP, 128, 0.5, 256.5), "rsqrt": (nm.SLOT_RSQRT, nm.FUNC_RSQRT, 64, 0.25, 4.0)}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


class Table:
    def __init__(self, func, n, lo, hi):
        k, b = nm.pwl_table_build(func, n, lo, hi)
        self.k, self.b, self.n, self.lo, self.hi = np.asarray(k, np.float64), np.asarray(b, np.float64), n, lo, hi

    def __call__(self, x, err=0.0):
        """The value at x and a bound on what it is off where x itself is off by up to err and the line is one fp32 FMA.  An x
        within err of a border may take the neighbour's line: the lines meet there up to the rounding of k and b."""
        x = np.asarray(x, np.float64)
        u = (x - self.lo) * self.n / (self.hi - self.lo)
        s = np.clip(np.floor(u), 0, self.n - 1).astype(int)
        # the index is one fp32 FMA: off by a few roundings of its terms, so up to a segment's neighbour when close
        slope = np.maximum(np.abs(self.k[s]), np.maximum(np.abs(self.k[np.maximum(s - 1, 0)]), np.abs(self.k[np.minimum(s + 1, self.n - 1)])))
        b = np.maximum(np.abs(self.b[s]), np.maximum(np.abs(self.b[np.maximum(s - 1, 0)]), np.abs(self.b[np.minimum(s + 1, self.n - 1)])))
        near = 4 * U * (np.abs(x) + abs(self.lo) + abs(self.hi))   # where the fp32 index may go to either side
        return self.k[s] * x + self.b[s], slope * (err + near) + 4 * U * (slope * np.abs(x) + b)


def load_tables(ctx):
    out = {}
    for name, (slot, func, n, lo, hi) in RANGES.items():
        ctx.load_function_table(slot, func, n, lo, hi)
        out[name] = Table(func, n, lo, hi)
    return out


def f64(t):
    return t.detach().double().cpu().numpy()


def check(got, ref, bound, dtype, what=""):
    """|got - ref| within `bound` (of the fp32 arithmetic) and one rounding to dtype."""
    got = f64(got)
    err, tol = np.abs(got - ref), bound + (np.abs(ref) + bound) * HALF_STEP[dtype] + TINY[dtype]
    bad = ~(err <= tol)
    assert not bad.any(), "%s: %d / %d outside, worst %.3g of its bound (%.6g for %.6g)" % (
        what, bad.sum(), bad.size, (err / tol)[bad].max() if np.isfinite(err[bad]).any() else math.nan, got[bad].ravel()[0], ref[bad].ravel()[0])


def attention(q, k, v, scale, exp_tab, recip_tab, p_step):
    """One head: q [d], k, v [n, d] in 64 bits.  p_step: relative rounding of a probability before it is multiplied into v.
    Sums in any order: at most n roundings of each term."""
    n, d = k.shape
    if n == 0:
        return np.zeros(d), np.zeros(d)
    s = scale * (k @ q)
    ds = (d + 4) * U * scale * (np.abs(k) @ np.abs(q))
    x = s - s.max()
    e, de = exp_tab(x, ds + ds.max() + U * np.abs(x))
    de = de + p_step * np.abs(e)
    total, dtotal = e.sum(), de.sum() + n * U * np.abs(e).sum()
    r, dr = recip_tab(total, dtotal)
    o = e @ v
    do = de @ np.abs(v) + (n + 4) * U * (np.abs(e) @ np.abs(v))
    return o * r, do * (abs(r) + dr) + np.abs(o) * dr + 2 * U * np.abs(o * r)


def rope(x, pos, cos_sin, gamma, eps, rot, pairs, tab):
    """x [T, heads, d] in 64 bits -> (y, bound).  The sum of squares takes at most 16 roundings of a term, the norm 4 more."""
    y, dy = x.copy(), np.zeros_like(x)
    if gamma is not None:
        var = (x * x).mean(-1, keepdims=True) + eps
        r, dr = tab(var, 18 * U * var)
        y = x * r * gamma
        dy = np.abs(x * gamma) * dr + 3 * U * np.abs(y)
    if rot:
        c, s = cos_sin[pos][:, None, :rot // 2], cos_sin[pos][:, None, rot // 2:]
        i = np.arange(rot // 2) * (2 if pairs else 1)
        j = i + (1 if pairs else rot // 2)
        a, b, da, db = y[..., i], y[..., j], dy[..., i], dy[..., j]
        u, w = a * c - b * s, b * c + a * s
        ac, bs, bc, as_ = np.abs(a * c), np.abs(b * s), np.abs(b * c), np.abs(a * s)
        y[..., i], y[..., j] = u, w
        dy[..., i] = da * np.abs(c) + db * np.abs(s) + 2 * U * (ac + bs)
        dy[..., j] = db * np.abs(c) + da * np.abs(s) + 2 * U * (bc + as_)
    return y, dy


def linear_w4(a, codes, scales, bias, residual, tab):
    """(y, bound) in 64 bits: every term takes at most K + 8 roundings of its size."""
    N, K = codes.shape[0], codes.shape[1] * 2
    c = np.empty((N, K))
    c[:, 0::2], c[:, 1::2] = (codes & 15).astype(np.float64) - 8, (codes >> 4).astype(np.float64) - 8
    w = c * np.repeat(scales, K // scales.shape[1], axis=1)
    y = a @ w.T
    dy = (K + 8) * U * (np.abs(a) @ np.abs(w).T)
    if bias is not None:
        y = y + bias
        dy = dy + U * np.abs(y)
    if tab is not None:
        y, dy = tab(y, dy)
    if residual is not None:
        y = y + residual
        dy = dy + U * np.abs(y)
    return y, dy


def plan(lengths, new, tables, free, count, page, max_tokens):
    """The step as a loop over requests; tables and free are changed in place."""
    B, width = tables.shape
    lengths, new = [int(x) for x in lengths], [int(x) for x in new]
    held = [-(-n // page) for n in lengths]
    same = {"lengths": lengths, "free_count": count, "token_start": [0] * (B + 1), "slots": [-1] * max_tokens, "positions": [0] * max_tokens}
    if any(n < 0 or n > width * page for n in lengths) or count < 0 or count > len(free):
        return 1, same
    back = sum(h for h, n in zip(held, new) if n < 0)
    if count + back > len(free):
        return 1, same
    add = [max(n, 0) for n in new]
    if any(n >= 0 and h + n > width * page for h, n in zip(lengths, new)) or sum(add) > max_tokens:
        return 2, same
    wanted = [0 if n < 0 else -(-(h + n) // page) - u for h, n, u in zip(lengths, new, held)]
    if sum(wanted) > count + back:
        return 8, same
    for i in range(B):
        if new[i] < 0:
            free[count:count + held[i]] = tables[i, :held[i]]
            count += held[i]
    slots, positions, start, out = [], [], [0], []
    for i in range(B):
        for e in range(held[i], held[i] + wanted[i]):
            count -= 1
            tables[i, e] = free[count]
        for p in range(lengths[i], lengths[i] + add[i]):
            slots.append(int(tables[i, p // page]) * page + p % page)
            positions.append(p)
        start.append(len(slots))
        out.append(0 if new[i] < 0 else lengths[i] + add[i])
    rest = max_tokens - len(slots)
    return 0, {"lengths": out, "free_count": count, "token_start": start, "slots": slots + [-1] * rest, "positions": positions + [0] * rest}
