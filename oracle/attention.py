"""Plain 64-bit oracle of the paged cache, attention over it and token importance
from queries and keys, with bounds on what 32-bit arithmetic may add.

Written from the formulas of ``include/mc_moe.h``: torch doubles on the CPU,
one sequence and one head at a time.  Test infrastructure only.
"""
from __future__ import annotations

import math

import torch

U24 = 2.0 ** -24          # half a step of fp32
BF = 2.0 ** -8            # half a step of bf16, relative


def unit(e4m3: bool) -> int:
    return 16 if e4m3 else 8


def offset(which: str, p: int, h: int, t: int, i: int, page: int, Hkv: int, D: int, U: int) -> int:
    """Element offset of (page, head, token of the page, dimension) in k or v,
    pages lying back to back."""
    base = p * Hkv * page * D
    if which == "k":
        return base + ((h * (page // 16) + t // 16) * (D // U) + i // U) * 16 * U + (t % 16) * U + i % U
    return base + ((h * (page // 16) + t // 16) * (16 // U) + (t % 16) // U) * D * U + i * U + t % U


def _offsets(which, pages, pos, h, page, Hkv, D, U):
    """[len(pos)][D] element offsets of whole rows."""
    t, i = (pos % page)[:, None], torch.arange(D)[None]
    base = (pages[pos // page].long() * Hkv * page * D)[:, None]
    if which == "k":
        return base + ((h * (page // 16) + t // 16) * (D // U) + i // U) * 16 * U + (t % 16) * U + i % U
    return base + ((h * (page // 16) + t // 16) * (16 // U) + (t % 16) // U) * D * U + i * U + t % U


def read(which, flat, pages, n, h, page, Hkv, D, U):
    """Rows 0 .. n-1 of a sequence's head as doubles [n][D] (flat: the cache array)."""
    at = _offsets(which, pages, torch.arange(n), h, page, Hkv, D, U)
    raw = flat.view(torch.uint8 if flat.element_size() == 1 else torch.int16)
    return raw[at.reshape(-1)].view(flat.dtype).double().view(n, D)


def write(which, flat, pages, pos, h, rows, page, Hkv, D, U):
    """Writes rows [len(pos)][D] (of the cache's type) at positions pos."""
    at = _offsets(which, pages, pos, h, page, Hkv, D, U)
    raw = torch.uint8 if flat.element_size() == 1 else torch.int16
    flat.view(raw)[at.reshape(-1)] = rows.contiguous().view(raw).reshape(-1)


def cap_error(s, cap):
    """What fp32 may add to capped scores s.  Caps to 64: cap - 2 cap u with u = 1 / (1 + e), e =
    exp(2 x / cap), is off by some 2^-23 cap whatever the score.  Above, the error is relative:
    from |x| = cap / 4 on cap (1 - 2 u), where e is off by 2 + 8 |x / cap| half steps (one step
    of exp2, 4 roundings in its argument), u by 1 - u of that and 3 (the sum, one step of the
    reciprocal), which is 5.6 of 1 - 2 u = 0.245 at x = -cap / 4, 23 half steps, and falls
    from there; 4 more are 1 - 2 u, the cap in the log2 domain and their product."""
    return 8 * U24 * cap if cap <= 64 else 28 * U24 * s.abs()


def scores(q, k, pos, scale, cap=0.0, window=0, slope=0.0, prefix=0):
    """(s [R][n] with -inf where a key is hidden, bound [R] on the fp32 error of a
    visible score).  The product's D terms, the scaling to the log2 domain, a
    difference of positions and the capped value are each rounded to fp32."""
    n, D = k.shape
    z = (q @ k.t()) * scale
    mag = (q.abs() @ k.abs().t()) * abs(scale)
    err = (D + 6) * U24 * mag
    if cap:
        z = cap * torch.tanh(z / cap)
        err = err + cap_error(z, cap)
    j = torch.arange(n)[None]
    i = torch.as_tensor(pos)[:, None]
    if slope:
        z = z + slope * (j - i)
        err = err + 4 * U24 * (slope * (j - i)).abs()
    seen = (j <= i) & ((j > i - window) if window else (j >= 0))
    seen = seen | ((j < prefix) & (i >= 0))
    s = torch.where(seen, z, torch.full_like(z, -math.inf))
    top = torch.where(seen, z.abs(), torch.zeros_like(z)).amax(1)
    err = torch.where(seen, err, torch.zeros_like(err)).amax(1) + 8 * U24 * top
    return s, err


def attend(q, k, v, pos, **kw):
    """(o [R][D], lse [R], tolerances of both): a row that sees nothing gets 0 and
    -inf.  With weights w and A = sum w |v|: the weights are off by twice the
    scores' error (numerator and sum), by 2^-8 from their rounding to bf16, and by
    2 n 2^-24 from the sums; the result is rounded once more."""
    n = k.shape[0]
    if n == 0:
        o, lse = torch.zeros_like(q), torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
        return o, lse, torch.zeros_like(o), torch.zeros_like(lse)
    s, err = scores(q, k, pos, **kw)
    m = s.amax(1)
    empty = m == -math.inf
    e = torch.exp(s - torch.where(empty, torch.zeros_like(m), m)[:, None])
    e = torch.where(s == -math.inf, torch.zeros_like(e), e)
    l = e.sum(1)
    w = e / torch.where(empty, torch.ones_like(l), l)[:, None]
    # only visible values count, whatever the others hold
    vis = s != -math.inf
    finite = torch.isfinite(v)
    o = w @ torch.where(finite, v, torch.zeros_like(v))
    if not finite.all():
        for j in torch.nonzero(~finite.all(1)).flatten().tolist():
            o = o + torch.where(vis[:, j:j + 1] & ~finite[j][None], w[:, j:j + 1] * v[j][None], torch.zeros_like(o))
    A = w @ torch.where(finite, v, torch.zeros_like(v)).abs()
    lse = torch.where(empty, torch.full_like(m, -math.inf), m + torch.log(l))
    rel = (2 * err + (2 * n + 64) * U24 + BF)[:, None]
    tol = rel * A + BF * (o.abs() + rel * A)
    tol_l = err + (n + 16) * U24 + 8 * U24 * (1 + torch.where(empty, torch.zeros_like(lse), lse).abs())
    return o, lse, tol, tol_l


def prepare(x, heads, D, weight, norm, eps, rot, pairs, rope):
    """(y [T][heads][D], bound): norm ("none", "head", "row") and rotation of rows
    x [T][heads * D] by the rows of rope [T][rot/2][2]."""
    T = x.shape[0]
    y = x.view(T, heads, D)
    W = 0
    if norm == "head":
        W = D
        y = y * weight / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
    elif norm == "row":
        W = heads * D
        y = y * weight.view(heads, D) / torch.sqrt((y * y).mean((1, 2), keepdim=True) + eps)
    mag = y.abs()
    if rot:
        c, s = rope[..., 0][:, None], rope[..., 1][:, None]
        a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if pairs else (y[..., :rot // 2], y[..., rot // 2:rot])
        ra, rb = a * c - b * s, a * s + b * c
        ma, mb = (a * c).abs() + (b * s).abs(), (a * s).abs() + (b * c).abs()
        y, mag = y.clone(), mag.clone()
        if pairs:
            y[..., 0:rot:2], y[..., 1:rot:2], mag[..., 0:rot:2], mag[..., 1:rot:2] = ra, rb, ma, mb
        else:
            y[..., :rot // 2], y[..., rot // 2:rot] = ra, rb
            mag[..., :rot // 2], mag[..., rot // 2:rot] = ma, mb
    return y, ((W + 24) * U24 if W or rot else 0.0) * mag


def importance(q, lse, k, x, L, g, Hkv, D, **kw):
    """(I [L], relative tolerance): queries q [L][Hq*D], lse [L][Hq], k a list of
    the key-value heads' keys [L][D]; slope: a list by query head."""
    slopes = kw.pop("slopes", None)
    sums = torch.zeros(L, dtype=torch.float64)
    worst = 0.0
    for h in range(Hkv * g):
        s, err = scores(q[:, h * D:(h + 1) * D], k[h // g], torch.arange(L),
                        slope=0.0 if slopes is None else float(slopes[h]), **kw)
        sums += torch.where(s == -math.inf, torch.zeros_like(s), torch.exp(s - lse[:, h:h + 1])).sum(0)
        worst = max(worst, float(err.max() + 8 * U24 * (1 + lse[:, h].abs().max())))
    norm = x.abs().sum(1)
    out = norm * sums / (Hkv * g) / (L - torch.arange(L)).double()
    return out, 1.01 * (worst + (L * g * Hkv + x.shape[1] + 64) * U24)
