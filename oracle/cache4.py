"""Plain 64-bit oracle of the 4-bit cache, a batch's tables and the selection of pages.

Written from the formulas of ``include/mc_moe.h``: torch on the CPU, loops over
requests, rows and heads.  Test infrastructure only.
"""
from __future__ import annotations

import math

import torch

from . import attention as oa

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
U24 = oa.U24


# ------------------------------------------------------------------ format --

def page_bytes(page: int, Hkv: int, D: int) -> int:
    return page * Hkv * D * 17 // 32


def code_place(which: str, h: int, t: int, i: int, page: int, D: int):
    """(byte of the page, half) of the code of token t of the page, dimension i."""
    B = h * (page // 16) + t // 16
    if which == "k":
        return B * 8 * D + (i // 32) * 256 + (t % 16) * 16 + (i % 32) // 2, i % 2
    return B * 8 * D + (i // 32) * 256 + (i % 16) * 16 + 8 * (i // 16 % 2) + (t % 16) // 2, t % 2


def scale_place(which: str, h: int, t: int, i: int, page: int, Hkv: int, D: int) -> int:
    """Byte of the page at which the scale of token t's dimension i lies."""
    z = Hkv * page * D // 2 + (h * (page // 16) + t // 16) * (D // 2)
    if which == "k":
        return z + (i // 32) * 16 + 4 * (t % 4) + t % 16 // 4
    return z + (i // 64) * 32 + 2 * (t % 16)


def nearest(x):
    """Codes (sign bit 8) of the levels nearest to x, ties to the even code."""
    a = x.abs()
    code = torch.zeros(x.shape, dtype=torch.int64)
    for c in range(7):
        border = (LEVELS[c] + LEVELS[c + 1]) / 2
        code += (a >= border) if c % 2 else (a > border)
    return code | torch.where(torch.signbit(x), 8, 0)


def _groups(y, n):
    b = y.double().reshape(*y.shape[:-1], y.shape[-1] // n, n)
    return b, b.abs().amax(-1)


def quantize_keys(y):
    """(codes [..][D], scale bytes [..][D / 32]) of keys."""
    b, m = _groups(y, 32)
    live = (m >= 2.0 ** -100) & (m <= 7 * 2.0 ** 125)
    e = torch.ceil(torch.log2(torch.where(live, m, torch.full_like(m, 7.0)) / 7))
    e = torch.where(m <= 7 * torch.exp2(e - 1), e - 1, torch.where(m > 7 * torch.exp2(e), e + 1, e))
    byte = torch.where(live, e + 127, torch.where(m < 2.0 ** -100, 0.0, 255.0)).long()
    codes = torch.where(live[..., None], nearest(b * torch.exp2(-e)[..., None]), 0)
    return codes.view(y.shape), byte


def six_bits(x):
    """Positive x rounded to 6 significant bits, ties to even."""
    m, e = torch.frexp(x)
    return torch.round(m * 64) / 64 * torch.exp2(e.double())


def quantize_values(v):
    """(codes [..][D], scales [..][D / 64] in 64 bits) of values."""
    b, m = _groups(v, 64)
    sixth = torch.tensor(1.0, dtype=torch.float32) / torch.tensor(6.0, dtype=torch.float32)
    live = (m >= 2.0 ** -100) & (m <= 7 * 2.0 ** 125)
    s = six_bits((torch.where(live, m, torch.ones_like(m)).float() * sixth).double())
    codes = torch.where(live[..., None], nearest(b / s[..., None]), 0)
    return codes.view(v.shape), torch.where(live, s, torch.where(m < 2.0 ** -100, 0.0, math.nan))


def values(which, codes, scale):
    """The numbers that codes [..][D] stand for; scale: bytes (k) or numbers (v)."""
    n = 32 if which == "k" else 64
    s = torch.where(scale == 255, math.nan, torch.exp2(scale.double() - 127)) if which == "k" else scale
    x = LEVELS[codes & 7] * torch.where(codes >= 8, -1.0, 1.0).double()
    return x * s.repeat_interleave(n, -1)


def _places(which, h, pos, page, Hkv, D):
    t, i = (pos % page)[:, None], torch.arange(D)[None]
    at, half = torch.broadcast_tensors(*code_place(which, h, t, i, page, D))
    return at, half, scale_place(which, h, t, torch.arange(0, D, 32 if which == "k" else 64)[None], page, Hkv, D)


def write(which, flat, pages, pos, h, codes, scale, page, Hkv, D):
    """Writes rows [len(pos)] of a head into the cache bytes flat [n_pages][bytes]."""
    if len(pos) == 0:
        return
    at, half, sc = _places(which, h, pos, page, Hkv, D)
    pg = pages[pos // page].long()[:, None]
    for hb in (0, 1):
        m = half == hb
        p, a, c = pg.expand_as(at)[m], at[m], codes[m].to(torch.uint8)
        # two tokens or two dimensions share a byte: one half at a time
        flat[p, a] = (flat[p, a] & (0xf0 if hb == 0 else 0x0f)) | (c << (4 * hb))
    if which == "k":
        flat[pg, sc] = scale.to(torch.uint8)
    else:
        raw = torch.where(torch.isnan(scale), 0x7fc0, scale.float().view(torch.int32) >> 16).to(torch.int16)
        raw = raw.view(*scale.shape, 1).view(torch.uint8)
        flat[pg, sc], flat[pg, sc + 1] = raw[..., 0], raw[..., 1]


def read(which, flat, pages, n, h, page, Hkv, D):
    """Rows 0 .. n-1 of a sequence's head as doubles [n][D]."""
    if n == 0:
        return torch.zeros((0, D), dtype=torch.float64)
    pos = torch.arange(n)
    at, half, sc = _places(which, h, pos, page, Hkv, D)
    pg = pages[pos // page].long()[:, None]
    codes = (flat[pg, at].long() >> (4 * half)) & 15
    if which == "k":
        return values("k", codes, flat[pg, sc].long())
    raw = torch.stack((flat[pg, sc], flat[pg, sc + 1]), -1).contiguous().view(torch.bfloat16).squeeze(-1)
    return values("v", codes, raw.double())


# ------------------------------------------------------------------ tables --

def reserve(want, past, free, n_free, table, page, T):
    """Lists of q_start, kv_len, positions, slots, and the stack's height left; table is filled in."""
    S, max_pages = len(want), table.shape[1]
    height = min(max(n_free, 0), len(free))
    P = R = taken = 0
    q_start, kv_len, positions, slots = [0], [], [], []
    for s in range(S):
        fits = want[s] >= 0 and past[s] >= 0 and past[s] + want[s] <= max_pages * page
        w = want[s] if fits else 0
        old = -(-past[s] // page)
        need = -(-(past[s] + w) // page) - old if fits else 0
        P, R = P + need, R + w
        n = w if R <= T and (need == 0 or P <= height) else 0
        if n:
            for i in range(need):
                table[s, old + i] = free[height - 1 - (P - need) - i]
            taken += need
        q_start.append(q_start[-1] + n)
        kv_len.append(past[s] + n)
        for t in range(n):
            p = past[s] + t
            positions.append(p)
            slots.append(int(table[s, p // page]) * page + p % page)
    positions += [-1] * (T - len(positions))
    slots += [-1] * (T - len(slots))
    return q_start, kv_len, positions, slots, height - taken


def release(done, past, free, n_free, table, page):
    """kv_len and the stack's height; free is filled in."""
    height = min(max(n_free, 0), len(free))
    kv_len = []
    for s in range(len(done)):
        if done[s] and past[s] > 0:
            for i in range(min(-(-past[s] // page), table.shape[1])):
                if height < len(free):
                    free[height] = int(table[s, i])
                height += 1
        kv_len.append(0 if done[s] else past[s])
    return kv_len, min(height, len(free))


# --------------------------------------------------------------- selection --

_127TH = torch.tensor(1.0, dtype=torch.float32) / torch.tensor(127.0, dtype=torch.float32)


def bounds(k):
    """(lo [D], hi [D] whole numbers, scale fp32) of a page's keys k [tokens][D]."""
    D = k.shape[1]
    lo, hi = torch.zeros(D), torch.zeros(D)
    for i in range(D):
        x = k[:, i][torch.isfinite(k[:, i])]
        if len(x):
            lo[i], hi[i] = float(x.min()), float(x.max())
    s = torch.maximum(lo.abs(), hi.abs()).max() * _127TH
    by = s if s > 0 else torch.tensor(1.0)
    return (lo / by).floor().clamp(-127, 127).long(), (hi / by).ceil().clamp(-127, 127).long(), s


def select(q, lo, hi, scale, pos, page, n_sel, first, last, window=0, negative=False):
    """Pages of a row: q [g][D] (fp32), lo and hi [pages][D], scale [pages]."""
    if pos < 0:
        return []
    end = pos // page
    begin = max(0, pos - window + 1) // page if window else 0
    if end - begin + 1 <= n_sel:
        return list(range(begin, end + 1))
    q = torch.where(torch.isfinite(q), -q if negative else q, torch.zeros_like(q))
    sq = q.abs().amax(1) * _127TH
    q8 = (q / torch.where(sq > 0, sq, torch.ones_like(sq))[:, None]).round().clamp(-127, 127).long()
    whole = q8.clamp(min=0) @ hi.t() + q8.clamp(max=0) @ lo.t()                  # [g][pages]
    score = (whole.float() * (sq[:, None] * scale[None])).amax(0)
    pages = list(range(begin, end + 1))
    kept = [p for p in pages if p < first or p > end - last]
    rest = sorted((p for p in pages if p not in kept), key=lambda p: (-float(score[p]), p))
    return sorted(kept + rest[:n_sel - len(kept)])


def attend_some(q, k, v, pos, times, **kw):
    """As attention.attend for one row q [1][D], key j counted times[j] times."""
    if k.shape[0] == 0:
        return torch.zeros_like(q), torch.full((1,), -math.inf, dtype=torch.float64), torch.zeros_like(q), \
            torch.zeros(1, dtype=torch.float64)
    s, err = oa.scores(q, k, torch.tensor([pos]), **kw)
    s = torch.where(times > 0, s + torch.log(times.clamp(min=1).double()), torch.full_like(s, -math.inf))
    if not bool((s > -math.inf).any()):
        return torch.zeros_like(q), torch.full((1,), -math.inf, dtype=torch.float64), torch.zeros_like(q), \
            torch.zeros(1, dtype=torch.float64)
    lse = torch.logsumexp(s, 1)
    w = torch.exp(s - lse[:, None])
    seen = w > 0
    vis = torch.where((s > -math.inf)[0][:, None], v, torch.zeros_like(v))
    o, A = w @ vis, w @ vis.abs()
    n = int(seen.sum())
    rel = (2 * err + (2 * n + 64) * U24 + oa.BF)[:, None]
    return o, lse, rel * A + oa.BF * (o.abs() + rel * A), err + (n + 16) * U24 + 8 * U24 * (1 + lse.abs())
