"""Workloads of a serving loop's cache: its tables, its 4-bit form, attention over selected pages.

Each case is one step that a serving program takes around the attention calls:

* ``tables``   ended requests give their pages back, running and new ones get
               theirs, with the batch's row starts, positions and slots;
* ``append``   norms and rotates new queries and keys and writes keys and values
               into a 4-bit cache; the new tokens are read back;
* ``decode``   attention of one new token a sequence over a 4-bit cache;
* ``prefill``  causal attention of prompts and chunks over it;
* ``sparse``   brings the bounds of the pages that the step touched up to date,
               selects pages for every query from the bounds, and attends to those.

``listed()`` gives the named cases, ``draw(rng)`` one more of the same ranges.
``run`` computes a case in its plain form (elementary torch operations), or, where
``own`` is true, with the package's calls.

Cache pages hold blocks of 16 tokens.  bf16 and e4m3, in units of 16 bytes (U = 8 or
16 elements): k[head][token / 16][d / U][token % 16][d % U], v[head][token / 16][token
% 16 / U][d][token % U].  e2m1 (two codes a byte, the first in the low half), all codes
of the page first:
    k[head][token / 16][d / 32][token % 16][d % 32]
    v[head][token / 16][d / 32][d % 16][d / 16 % 2][token % 16]
then the scales: of keys one byte for 32 dimensions, 2^(byte - 127) (255: NaN),
[head][token / 16][d / 32][token % 4][token % 16 / 4]; of values bf16 for 64 dimensions,
[head][token / 16][d / 64][token % 16].
"""
from __future__ import annotations

import math
import random

import torch

own = False

_NINF = float("-inf")
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)       # of e2m1
_LEAST = 2.0 ** -100                                      # groups of smaller values are 0
_MOST = 7 * 2.0 ** 125                                    # groups of larger ones are NaN
_EPS = float(torch.tensor(1e-5, dtype=torch.float32))


def _heads(Hq, Hkv, D, page, kv):
    return dict(Hq=Hq, Hkv=Hkv, D=D, page=page, kv=kv)


_MIXTRAL = (32, 8, 128)      # the attention heads that go with the Mixtral-shaped layers
_OLMOE = (16, 16, 128)       # and with the OLMoE-shaped ones


def _tables(name, S, page, new, past, ended, short, mix):
    return dict(name=name, kind="tables", S=S, page=page, new_lo=new[0], new_hi=new[1], past_lo=past[0],
                past_hi=past[1], ended=ended, short=short, mix=mix)


def _append(name, heads, S, new, past, norm, rot, pairs, mix):
    return dict(name=name, kind="append", S=S, new_lo=new[0], new_hi=new[1], past_lo=past[0], past_hi=past[1],
                norm=norm, rot=rot, pairs=pairs, mix=mix, **heads)


def _attention(name, kind, heads, S, new, past, mix, window=0, cap=0.0, slopes=False, prefix=0):
    return dict(name=name, kind=kind, S=S, new_lo=new[0], new_hi=new[1], past_lo=past[0], past_hi=past[1],
                window=window, cap=cap, slopes=slopes, prefix=prefix, mix=mix, **heads)


def _sparse(name, heads, S, new, past, n_sel, first, last, mix, window=0, cap=0.0):
    return dict(_attention(name, "sparse", heads, S, new, past, mix, window, cap), n_sel=n_sel, first=first, last=last)


def listed():
    return [
        # one decode step of 64 conversations, a few of them just ended: all latency
        _tables("tables_step_64", 64, 16, (1, 1), (100, 8000), 0.06, False, 1),
        # a large batch of short requests, prompts and decoding ones; the pool runs out
        _tables("tables_batch_2048", 2048, 32, (1, 60), (0, 2000), 0.2, True, 2),
        # one decode step of 64 sequences: scattered single tokens
        _append("append_step_64", _heads(*_MIXTRAL, 16, "e2m1"), 64, (1, 1), (100, 600), "none", 128, False, 3),
        # prompts of a few thousand tokens, norms over the whole projection
        _append("append_prompts", _heads(*_OLMOE, 64, "e2m1"), 5, (700, 2900), (0, 33), "row", 128, False, 4),
        # interactive decoding of one short conversation
        _attention("decode_one", "decode", _heads(*_OLMOE, 16, "e2m1"), 1, (1, 1), (776, 776), 5),
        # batched decoding, ragged lengths
        _attention("decode_batch_48", "decode", _heads(*_MIXTRAL, 16, "e2m1"), 48, (1, 1), (300, 8191), 6),
        # a few sequences over long documents
        _attention("decode_long", "decode", _heads(*_MIXTRAL, 256, "e2m1"), 4, (1, 1), (50000, 131071), 7),
        # short ragged prompts, some of one token, heads of 64
        _attention("prefill_short", "prefill", _heads(32, 8, 64, 16, "e2m1"), 9, (1, 333), (0, 50), 8),
        # chunks of long prompts
        _attention("prefill_chunks", "prefill", _heads(*_MIXTRAL, 128, "e2m1"), 2, (1500, 2048), (5000, 8192), 9),
        # one conversation over a long document
        _sparse("sparse_one", _heads(*_MIXTRAL, 64, "bf16"), 1, (1, 1), (33333, 33333), 32, 1, 2, 10),
        # batched decoding over long documents
        _sparse("sparse_batch_16", _heads(*_MIXTRAL, 64, "bf16"), 16, (1, 1), (20000, 131071), 64, 1, 2, 11),
        # chunks of two prompts, each token its own pages, a 4-bit cache
        _sparse("sparse_chunks", _heads(*_MIXTRAL, 64, "e2m1"), 2, (100, 128), (9000, 16384), 32, 1, 2, 12),
    ]


def _log(rng, lo, hi):
    """A whole number spread evenly over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tables", "append", "decode", "prefill", "sparse"])
    mix = rng.randrange(1 << 20)
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "tables":
        S = _log(rng, 1, 2048)
        hi = _log(rng, 1, max(1, min(2900, 65536 // S)))
        c = _tables("", S, page, (rng.randint(0, hi), hi), (0, _log(rng, 1, 4000)), rng.choice([0.0, 0.1, 0.5]),
                    rng.random() < 0.3, mix)
        c.pop("name")
        return c
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8, 16] if D == 128 else [2, 4, 8, 16, 32])
    g = rng.choice([1, 2, 3, 4, 5, 8])
    if Hkv * g > 64:
        g = max(1, 32 // Hkv)
    kv = rng.choice(["bf16", "e4m3", "e2m1"]) if kind == "sparse" else "e2m1"
    heads = _heads(Hkv * g, Hkv, D, page, kv)
    extra = dict(window=rng.choice([0, 0, _log(rng, 32, 5000)]), cap=rng.choice([0.0, 0.0, 20.0, 50.0]))
    if kind == "append":
        S = _log(rng, 1, 128)
        hi = _log(rng, 1, max(1, min(2900, 12000 // S)))
        c = _append("", heads, S, (rng.randint(1, hi), hi), (0, rng.choice([0, 33, 500])),
                    rng.choice(["none", "head", "row"]), rng.choice([D, D, D // 2, 0]), rng.random() < 0.3, mix)
    elif kind == "decode":
        S = _log(rng, 1, 128)
        hi = _log(rng, 1, min(131071, max(1, 2000000 // (S * max(1, Hkv * D // 256)))))
        c = _attention("", kind, heads, S, (1, 1), (rng.randint(0, hi), hi), mix, prefix=rng.choice([0, 0, 5]),
                       slopes=rng.random() < 0.3, **extra)
    elif kind == "prefill":
        S = _log(rng, 1, 12)
        hi = _log(rng, 1, max(8, min(2048, 4000 // S)))
        past = rng.choice([0, 0, _log(rng, 1, 4000)])
        c = _attention("", kind, heads, S, (rng.randint(1, hi), hi), (0, past), mix, prefix=rng.choice([0, 0, 70]),
                       slopes=rng.random() < 0.3, **extra)
    else:
        n_sel = _log(rng, 2, max(2, 4096 // page))
        rows = max(1, 262144 // (n_sel * page * max(1, Hkv * D // 1024)))
        S = _log(rng, 1, min(32, rows))
        hi = _log(rng, 1, max(1, min(128, rows // S)))
        past = _log(rng, 1, min(131071, max(1, 1200000 // (S * max(1, Hkv * D // 256)))))
        first = rng.choice([0, 1])
        c = _sparse("", heads, S, (rng.randint(1, hi), hi), (rng.randint(0, past), past), n_sel, first,
                    rng.randint(1, min(3, n_sel - first)), mix, **extra)
    c.pop("name", None)
    return c


def _lengths(case):
    """(new tokens, tokens before them) of each sequence; the first sequence has the most of both."""
    r = random.Random(case["mix"])
    n = [(r.randint(case["new_lo"], case["new_hi"]), r.randint(case["past_lo"], case["past_hi"]))
         for _ in range(case["S"])]
    n[0] = (case["new_hi"], case["past_hi"])
    return n


# ------------------------------------------------------------------ inputs --

def _tables_state(case, seed):
    """The requests' lengths, the pages that they hold, and the pool of free ones."""
    dev = torch.device("cuda")
    S, page = case["S"], case["page"]
    n = _lengths(case)
    r = random.Random(case["mix"] + 1)            # which end is the case's, the pages are the seed's
    ended = [0] + [int(r.random() < case["ended"]) for _ in range(S - 1)]
    past = [b for _, b in n]
    want = [0 if e else a for (a, _), e in zip(n, ended)]
    held = [-(-b // page) for b in past]
    after = [-(-(a + b) // page) for a, b in zip(want, past)]
    need = sum(a - h for a, h in zip(after, held))
    spare = need // 2 if case["short"] else need + 1 + S // 4
    n_pages = sum(held) + spare
    order = list(range(n_pages))
    random.Random(seed).shuffle(order)
    # rows are as long as the longest request, with a page to spare
    max_pages = max(after + held) + 1
    table = torch.full((S, max_pages), -1, dtype=torch.int32)
    table[torch.repeat_interleave(torch.arange(S), torch.tensor(held)), torch.cat([torch.arange(h) for h in held])] = \
        torch.tensor(order[:sum(held)], dtype=torch.int32)
    free = torch.full((n_pages,), -1, dtype=torch.int32)
    free[:spare] = torch.tensor(order[sum(held):], dtype=torch.int32)

    def i32(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    T = max(1, sum(want))
    st = dict(case=case, S=S, T=T, want=i32(want), past=i32(past), ended=i32(ended).to(torch.uint8),
              table=table.to(dev), free=free.to(dev), n_free=i32([spare]), n_free1=i32([0]), n_free2=i32([0]),
              len1=i32([0] * S), kv_len=i32([0] * S), q_start=i32([0] * (S + 1)), positions=i32([0] * T),
              slots=torch.zeros(T, dtype=torch.int64, device=dev))
    if own:
        import paper_2410_06270_amd as mc
        st["pool0"] = mc.KVPool(page, st["free"], st["n_free"], st["n_free1"])
        st["pool1"] = mc.KVPool(page, st["free"], st["n_free1"], st["n_free2"])
        st["batch1"] = mc.KVBatch(st["len1"], st["table"])
        st["batch"] = mc.KVBatch(st["kv_len"], st["table"], q_start=st["q_start"], T=T)
        st["ws"] = torch.empty(mc.kv_tables_workspace(S), dtype=torch.uint8, device=dev)
    return st


def prepare(case, seed):
    """The projections' outputs, the cache with its page table, and what a
    program keeps beside them: norm weights, the rotation table, slopes, page
    bounds, and the buffers that a call writes."""
    if case["kind"] == "tables":
        return _tables_state(case, seed)
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    Hq, Hkv, D, page, kind = case["Hq"], case["Hkv"], case["D"], case["page"], case["kind"]
    n = _lengths(case)
    S, T = len(n), sum(a for a, _ in n)
    used = [-(-(a + b) // page) for a, b in n]
    n_pages = sum(used) + 3
    st = dict(case=case, S=S, T=T, n_pages=n_pages, max_new=max(a for a, _ in n), max_len=max(a + b for a, b in n))
    q_start = [0]
    for a, _ in n:
        q_start.append(q_start[-1] + a)
    st["q_start"] = torch.tensor(q_start, dtype=torch.int32, device=dev)
    st["kv_len"] = torch.tensor([a + b for a, b in n], dtype=torch.int32, device=dev)
    order = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32)
    table = torch.zeros((S, max(used)), dtype=torch.int32, device=dev)
    rows = torch.repeat_interleave(torch.arange(S), torch.tensor(used)).to(dev)
    cols = torch.cat([torch.arange(u) for u in used]).to(dev)
    table[rows, cols] = order[:sum(used)]
    st["table"] = table

    # keys share one direction with the queries, each token to its own degree and pages
    # to theirs, and the first key draws the most: attention with a sink and a heavy tail
    kv = case["kv"]
    u = randn(Hkv, D)
    u = u / u.norm(dim=-1, keepdim=True)
    k, v = randn(n_pages, Hkv, page, D), randn(n_pages, Hkv, page, D)
    pull = torch.exp(0.8 * randn(n_pages, 1, page, 1) + 0.5 * randn(n_pages, Hkv, 1, 1))
    pull[table[:, 0].long(), :, 0] = 9.0
    k += pull * u.view(1, Hkv, 1, D)
    del pull
    st["k_scale"] = st["v_scale"] = None
    if kv == "e4m3":
        st["k_scale"] = 0.02 * torch.exp(0.3 * randn(Hkv))
        st["v_scale"] = 0.01 * torch.exp(0.3 * randn(Hkv))
        k = (k / st["k_scale"].view(1, Hkv, 1, 1)).clamp(-448, 448)
        v = (v / st["v_scale"].view(1, Hkv, 1, 1)).clamp(-448, 448)
    if kv == "e2m1":
        kind_t = torch.float4_e2m1fn_x2
        st["k_cache"], st["v_cache"] = _pages_k(*_quantize_keys(k)), _pages_v(*_quantize_values(v.to(torch.bfloat16)))
    else:
        kind_t = torch.float8_e4m3fn if kv == "e4m3" else torch.bfloat16
        U = 16 if kv == "e4m3" else 8
        k = k.view(n_pages, Hkv, page // 16, 16, D // U, U).transpose(3, 4)
        v = v.view(n_pages, Hkv, page // 16, 16 // U, U, D).transpose(4, 5)
        st["k_cache"], st["v_cache"] = (a.to(kind_t).contiguous().view(n_pages, -1) for a in (k, v))
    del k, v

    if kind == "append":
        # q, k and v lie side by side, as one projection writes them
        st["qkv"] = randn(T, (Hq + 2 * Hkv) * D).to(torch.bfloat16)
        st["q_out"] = torch.empty((T, Hq * D), dtype=torch.bfloat16, device=dev)
        st["k_out"] = torch.empty((T, Hkv * D), dtype=torch.bfloat16, device=dev)
        st["v_out"] = torch.empty((T, Hkv * D), dtype=torch.bfloat16, device=dev)
        rot = case["rot"]
        if rot:
            at = torch.arange(st["max_len"], dtype=torch.float64, device=dev)[:, None]
            ang = at * (1e6 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=dev) / rot))
            st["rope"] = torch.stack((ang.cos(), ang.sin()), -1).float().contiguous()
        else:
            st["rope"] = None
        wide = case["norm"] == "row"
        for name, h in (("q_norm", Hq), ("k_norm", Hkv)):
            st[name] = None if case["norm"] == "none" else \
                (1 + 0.1 * randn(h * D if wide else D)).to(torch.bfloat16)
    else:
        q = randn(T, Hkv, Hq // Hkv, D) + 1.5 * u.view(1, Hkv, 1, D)
        st["q"] = q.to(torch.bfloat16).view(T, Hq * D)
        st["scale"] = 1.0 / math.sqrt(D)
        h = torch.arange(1, Hq + 1, device=dev, dtype=torch.float32)
        st["slopes"] = torch.exp2(-8.0 * h / Hq) if case["slopes"] else None
        st["prefix"] = torch.full((S,), case["prefix"], dtype=torch.int32, device=dev) if case["prefix"] else None
        st["o"] = torch.empty((T, Hq * D), dtype=torch.bfloat16, device=dev)
        st["lse"] = torch.empty((T, Hq), dtype=torch.float32, device=dev)
    if kind == "sparse":
        # the bounds of all pages as the steps before left them
        st["bounds"] = torch.zeros((n_pages, Hkv, 2, D), dtype=torch.int8, device=dev)
        st["bound_scale"] = torch.zeros((n_pages, Hkv), dtype=torch.float32, device=dev)
        held = torch.tensor([min(page, max(0, b - i * page)) for (a, b), m in zip(n, used) for i in range(m)], device=dev)
        for i in range(0, sum(used), 2048):
            _plain_summarize(st, table[rows, cols][i:i + 2048].long(), held[i:i + 2048])
        st["sel"] = torch.full((T, Hkv, case["n_sel"]), -1, dtype=torch.int32, device=dev)
        st["count"] = torch.zeros((T, Hkv), dtype=torch.int32, device=dev)
    if own:      # the descriptors and the workspace, which a program keeps over all its steps
        import paper_2410_06270_amd as mc
        st["cache"] = mc.KVCache(n_pages, page, Hkv, D, dtype=kind_t, k=st["k_cache"], v=st["v_cache"],
                                 k_scale=st["k_scale"], v_scale=st["v_scale"])
        st["batch"] = mc.KVBatch(st["kv_len"], table, q_start=st["q_start"], T=T, max_len=st["max_len"])
        if kind == "append":
            st["prep"] = mc.QKPrep(rope=st["rope"], rope_pairs=case["pairs"], q_norm=st["q_norm"], k_norm=st["k_norm"],
                                   norm_row=case["norm"] == "row", eps=1e-5)
            return st
        st["attn"] = mc.Attention(Hq, st["scale"], softcap=case["cap"], window=case["window"], slopes=st["slopes"],
                                  prefix=st["prefix"])
        need = mc.attn_workspace(T, Hq, Hkv, D)
        if kind == "sparse":
            st["summary"] = mc.KVSummary(st["cache"], bounds=st["bounds"], scale=st["bound_scale"])
            need = max(need, mc.attn_select_workspace(T, Hkv, max(used)))
        st["ws"] = torch.empty(need, dtype=torch.uint8, device=dev)
    return st


# ------------------------------------------------------------- 4-bit cache --

def _pow2(e):
    """2^e of whole e, exactly, in 64 bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _nearest(x):
    """Codes 0 .. 7 of the levels nearest to x >= 0, ties to the even code (NaN: 0)."""
    return ((x > 0.25).to(torch.uint8) + (x >= 0.75) + (x > 1.25) + (x >= 1.75) + (x > 2.5) + (x >= 3.5) + (x > 5.0))


def _quantize_keys(y):
    """Codes [..][D] and scale bytes [..][D / 32] of keys y [..][D]: 32 dimensions share
    2^e, e the least with max |y| <= 7 * 2^e."""
    D = y.shape[-1]
    b = y.reshape(*y.shape[:-1], D // 32, 32)
    most = b.abs().amax(-1)
    ok = most <= _MOST
    m, k = torch.frexp(torch.where(ok, most, torch.ones_like(most)))
    e = k - 3 + (m > 0.875)
    zero = most < _LEAST
    byte = torch.where(zero, torch.zeros_like(e), torch.where(ok, e + 127, torch.full_like(e, 255))).to(torch.uint8)
    x = b.abs() * _pow2(-e)[..., None].to(b.dtype)
    code = _nearest(x) + 8 * (b < 0).to(torch.uint8)
    code = torch.where((zero | ~ok)[..., None], torch.zeros_like(code), code)
    return code.view(*y.shape), byte


def _quantize_values(v):
    """Codes [..][D] and scales [..][D / 64] (bf16) of values v [..][D] (bf16): 64 dimensions
    share s, max |v| / 6 rounded to 6 significant bits."""
    D = v.shape[-1]
    b = v.double().reshape(*v.shape[:-1], D // 64, 64)
    most = b.abs().amax(-1)
    ok = most <= _MOST
    bits = (most.float() / 6).view(torch.int32)
    bits = (bits + 0x1ffff + ((bits >> 18) & 1)) & ~0x3ffff
    s = bits.view(torch.float32)
    zero = most < _LEAST
    s = torch.where(zero, torch.zeros_like(s), torch.where(ok, s, torch.full_like(s, math.nan)))
    x = b.abs() / torch.where(zero | ~ok, torch.ones_like(s), s).double()[..., None]
    code = _nearest(x) + 8 * (b < 0).to(torch.uint8)
    code = torch.where((zero | ~ok)[..., None], torch.zeros_like(code), code)
    return code.view(*v.shape), s.to(torch.bfloat16)


def _pages_k(code, byte):
    """Pages [n][bytes] of key codes [n][Hkv][page][D] and their scale bytes."""
    n, Hkv, page, D = code.shape
    c = code.view(n, Hkv, page // 16, 16, D // 32, 32).transpose(3, 4)
    c = (c[..., 0::2] | (c[..., 1::2] << 4)).reshape(n, -1)
    s = byte.view(n, Hkv, page // 16, 4, 4, D // 32).permute(0, 1, 2, 5, 4, 3).reshape(n, -1)
    return torch.cat((c, s), 1)


def _pages_v(code, scale):
    n, Hkv, page, D = code.shape
    c = code.view(n, Hkv, page // 16, 16, D // 32, 2, 16).permute(0, 1, 2, 4, 6, 5, 3)
    c = (c[..., 0::2] | (c[..., 1::2] << 4)).reshape(n, -1)
    s = scale.view(n, Hkv, page // 16, 16, D // 64).transpose(3, 4).contiguous().view(n, -1).view(torch.uint8)
    return torch.cat((c, s), 1)


def _levels(code):
    t = torch.tensor(_LEVELS + tuple(-x for x in _LEVELS), device=code.device)
    return t[code.long()]


def _values_of(st, pages):
    """Keys and values [..][Hkv][page][D] (fp32) of pages [..]."""
    c = st["case"]
    Hkv, D, page = c["Hkv"], c["D"], c["page"]
    lead = tuple(pages.shape)
    k, v = (st[a].view(torch.uint8)[pages] for a in ("k_cache", "v_cache"))
    B = page // 16
    if c["kv"] != "e2m1":
        kt = st["k_cache"].dtype
        U = 16 // st["k_cache"].element_size()
        k = k.view(kt).view(*lead, Hkv, B, D // U, 16, U).float().transpose(-3, -2).reshape(*lead, Hkv, page, D)
        v = v.view(kt).view(*lead, Hkv, B, 16 // U, D, U).float().transpose(-2, -1).reshape(*lead, Hkv, page, D)
        return k, v
    cut = Hkv * page * D // 2
    ck, cv = (torch.stack((a[..., :cut] & 15, a[..., :cut] >> 4), -1) for a in (k, v))
    ck = _levels(ck.view(*lead, Hkv, B, D // 32, 16, 32).transpose(-3, -2)).reshape(*lead, Hkv, page, D // 32, 32)
    i = len(lead)
    cv = _levels(cv.view(*lead, Hkv, B, D // 32, 16, 2, 16).permute(*range(i), i, i + 1, i + 5, i + 2, i + 4, i + 3))
    sk = k[..., cut:].view(*lead, Hkv, B, D // 32, 4, 4).permute(*range(i), i, i + 1, i + 4, i + 3, i + 2)
    sk = sk.reshape(*lead, Hkv, page, D // 32, 1).int()
    sk = torch.where(sk == 255, math.nan, _pow2(sk - 127)).float()
    sv = v[..., cut:].contiguous().view(torch.bfloat16).view(*lead, Hkv, B, D // 64, 16).float()
    sv = sv.transpose(-2, -1).reshape(*lead, Hkv, page, D // 64, 1)
    cv = cv.reshape(*lead, Hkv, page, D // 64, 64)
    return (ck * sk).reshape(*lead, Hkv, page, D), (cv * sv).reshape(*lead, Hkv, page, D)


# -------------------------------------------------------------- plain form --

def _plain_tables(st):
    S, T, page = st["S"], st["T"], st["case"]["page"]
    table, free = st["table"], st["free"]
    max_pages = table.shape[1]
    past, ended = st["past"].long(), st["ended"].bool()
    col = torch.arange(max_pages, device="cuda")
    # ended requests push their pages
    held = torch.where(ended, (past + page - 1) // page, torch.zeros_like(past))
    start = torch.cumsum(held, 0) - held
    n_free = st["n_free"].long()
    gone = col < held[:, None]
    at = torch.where(gone, n_free + start[:, None] + col, torch.full_like(col, free.numel()))
    padded = torch.cat((free, free.new_zeros(1)))
    padded[at.reshape(-1)] = table.reshape(-1)
    free.copy_(padded[:-1])
    n_free1 = n_free + held.sum()
    past = torch.where(ended, torch.zeros_like(past), past)
    # the others pop theirs
    want = st["want"].long()
    fits = (want >= 0) & (past >= 0) & (past + want <= max_pages * page)
    want = torch.where(fits, want, torch.zeros_like(want))
    old = (past + page - 1) // page
    need = torch.where(fits, (past + want + page - 1) // page - old, torch.zeros_like(past))
    pages, rows = torch.cumsum(need, 0), torch.cumsum(want, 0)
    granted = (rows <= T) & ((need == 0) | (pages <= n_free1))
    take, new = torch.where(granted, need, torch.zeros_like(need)), torch.where(granted, want, torch.zeros_like(want))
    i = col - old[:, None]
    mine = (i >= 0) & (i < take[:, None])
    src = torch.where(mine, n_free1 - 1 - ((pages - need)[:, None] + i), torch.zeros_like(i))
    table.copy_(torch.where(mine, free[src], table))
    q_start = torch.cat((new.new_zeros(1), torch.cumsum(new, 0)))
    row = torch.arange(T, device="cuda")
    seq = torch.searchsorted(q_start[1:], row, right=True).clamp(max=S - 1)
    live = row < q_start[S]
    pos = torch.where(live, past[seq] + row - q_start[seq], torch.full_like(row, -1))
    slot = torch.where(live, table[seq, (pos // page).clamp(min=0)].long() * page + pos % page, torch.full_like(row, -1))
    return (q_start.int(), (past + new).int(), table, free, (n_free1 - take.sum()).int(), pos.int(), slot)


def _rows(st):
    """The sequence and the place among its new tokens of each packed row."""
    t = torch.arange(st["T"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(st["q_start"], t, right=True).long() - 1
    return seq, t.long() - st["q_start"].long()[seq]


def _positions(st):
    seq, r = _rows(st)
    q_start = st["q_start"].long()
    return seq, (st["kv_len"].long() - (q_start[1:] - q_start[:-1]))[seq] + r


def _plain_append(st):
    c = st["case"]
    Hq, Hkv, D, page, rot, T = c["Hq"], c["Hkv"], c["D"], c["page"], c["rot"], st["T"]
    q, k, v = st["qkv"].split((Hq * D, Hkv * D, Hkv * D), 1)
    seq, pos = _positions(st)

    # keys in 64 bits: their codes are decided at borders
    def finish(a, h, w):
        a = a.reshape(T, h, D)
        if c["norm"] == "head":
            a = a * w.to(a.dtype) / (a.square().mean(-1, keepdim=True) + _EPS).sqrt()
        elif c["norm"] == "row":
            a = a * w.to(a.dtype).view(h, D) / (a.square().mean((1, 2), keepdim=True) + _EPS).sqrt()
        if rot:
            cs, sn = (st["rope"][pos, :, i][:, None, :].to(a.dtype) for i in (0, 1))
            b = a[..., :rot]
            x, y = (b[..., 0::2], b[..., 1::2]) if c["pairs"] else (b[..., :rot // 2], b[..., rot // 2:])
            x, y = x * cs - y * sn, x * sn + y * cs
            b = torch.stack((x, y), -1).flatten(-2) if c["pairs"] else torch.cat((x, y), -1)
            a = torch.cat((b, a[..., rot:]), -1)
        return a

    q = finish(q.float(), Hq, st["q_norm"]).to(torch.bfloat16).view(T, Hq * D)
    kc, kb = _quantize_keys(finish(k.double(), Hkv, st["k_norm"]))
    vc, vs = _quantize_values(v.reshape(T, Hkv, D))
    pg, blk, tok = st["table"][seq, pos // page].long(), pos % page // 16, pos % 16
    kp, vp = st["k_cache"], st["v_cache"]
    cut = Hkv * page * D // 2
    h = torch.arange(Hkv, device="cuda")
    at = (h * (page // 16) + blk[:, None]) * 8 * D                # [T][Hkv]
    i = torch.arange(D // 2, device="cuda")
    pair = kc[..., 0::2] | (kc[..., 1::2] << 4)
    kp[pg[:, None, None], at[..., None] + (i // 16 * 256 + i % 16) + (tok * 16)[:, None, None]] = pair
    j = torch.arange(D // 32, device="cuda")
    kp[pg[:, None, None], (cut + at // 16)[..., None] + j * 16 + (tok % 4 * 4 + tok // 4)[:, None, None]] = kb
    d = torch.arange(D, device="cuda")
    place = at[..., None] + (d // 32 * 256 + d % 16 * 16 + d // 16 % 2 * 8) + (tok // 2)[:, None, None]
    for half in (0, 1):       # of a byte: even tokens, then odd ones
        m = tok % 2 == half
        p, w = (pg[m][:, None, None], place[m])
        vp[p, w] = (vp[p, w] & (0xf0 if half == 0 else 0x0f)) | (vc[m] << (4 * half))
    e = torch.arange(D // 64, device="cuda")
    vp.view(torch.int16)[pg[:, None, None], ((cut + at // 16) // 2)[..., None] + e * 16 + tok[:, None, None]] = \
        vs.view(torch.int16)
    sk = torch.where(kb == 255, math.nan, _pow2(kb.int() - 127)).float()
    k = _levels(kc).view(T, Hkv, D // 32, 32) * sk[..., None]
    v = _levels(vc).view(T, Hkv, D // 64, 64) * vs.float()[..., None]
    return q, k.view(T, Hkv * D).to(torch.bfloat16), v.view(T, Hkv * D).to(torch.bfloat16)


def _scored(st, s, pos, j, heads):
    """Capped and masked scores; pos and j broadcast to s, heads is the shape of the slopes in it."""
    c = st["case"]
    s *= st["scale"]
    if c["cap"]:
        s = torch.tanh(s / c["cap"]) * c["cap"]
    if st["slopes"] is not None:
        s += st["slopes"].view(heads) * (j - pos).float()
    seen = j <= pos
    if c["window"]:
        seen = seen & (j > pos - c["window"])
    return s, seen


def _softmax(s):
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == _NINF, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    return p, l, m + l.log()


def _plain_attention(st):
    c = st["case"]
    S, R, Hq, Hkv, D = st["S"], st["max_new"], c["Hq"], c["Hkv"], c["D"]
    g = Hq // Hkv
    k, v = (a.transpose(1, 2).reshape(S, Hkv, -1, D) for a in _values_of(st, st["table"].long()))
    Lk = k.shape[2]
    seq, r = _rows(st)
    q = torch.zeros((S, R, Hkv, g, D), dtype=torch.float32, device="cuda")
    q[seq, r] = st["q"].float().view(-1, Hkv, g, D)
    q = q.permute(0, 2, 3, 1, 4).reshape(S, Hkv, g * R, D)
    s = torch.matmul(q, k.transpose(2, 3)).view(S, Hkv, g, R, Lk)
    del k
    kv_len, q_start = st["kv_len"].long(), st["q_start"].long()
    pos = (kv_len - (q_start[1:] - q_start[:-1]))[:, None] + torch.arange(R, device="cuda")
    j = torch.arange(Lk, device="cuda")
    s, seen = _scored(st, s, pos[:, None, None, :, None], j, (1, Hkv, g, 1, 1))
    if st["prefix"] is not None:
        seen = seen | (j < st["prefix"][:, None, None, None, None])
    s.masked_fill_(~(seen & (j < kv_len[:, None, None, None, None])), _NINF)
    p, l, lse = _softmax(s)
    v = v * (j < kv_len[:, None])[:, None, :, None]
    o = torch.matmul(p.view(S, Hkv, g * R, Lk), v).view(S, Hkv, g, R, -1)
    o = torch.where(l > 0, o / l, torch.zeros_like(o))
    o = o.permute(0, 3, 1, 2, 4)[seq, r].reshape(-1, Hq * D)
    return o.to(torch.bfloat16), lse.squeeze(-1).permute(0, 3, 1, 2)[seq, r].reshape(-1, Hq)


def _plain_summarize(st, pages, held):
    """Bounds of the first `held` keys of each page."""
    k, _ = _values_of(st, pages)                                             # [n][Hkv][page][D]
    out = ~((torch.arange(k.shape[2], device="cuda") < held[:, None])[:, None, :, None] & torch.isfinite(k))
    lo, hi = k.masked_fill(out, math.inf).amin(2), k.masked_fill(out, _NINF).amax(2)
    lo, hi = (torch.where(torch.isinf(a), torch.zeros_like(a), a) for a in (lo, hi))
    s = torch.maximum(lo.abs(), hi.abs()).amax(-1) / 127
    d = torch.where(s > 0, s, torch.ones_like(s))[..., None]
    st["bounds"][pages] = torch.stack(((lo / d).floor(), (hi / d).ceil()), 2).clamp(-127, 127).to(torch.int8)
    st["bound_scale"][pages] = s


def _plain_select(st):
    c = st["case"]
    T, Hkv, D, page, N = st["T"], c["Hkv"], c["D"], c["page"], c["n_sel"]
    g = c["Hq"] // Hkv
    seq, pos = _positions(st)
    q = st["q"].float().view(T, Hkv, g, D)
    sq = q.abs().amax(-1) / 127
    q8 = (q / torch.where(sq > 0, sq, torch.ones_like(sq))[..., None]).round().clamp(-127, 127)
    # whole numbers below 2^24 in all partial sums: exact in fp32
    P = st["table"].shape[1]
    at = st["table"].long()
    b = st["bounds"][at].float().permute(0, 2, 3, 4, 1)                      # [S][Hkv][2][D][P]
    both = torch.cat((q8.clamp(max=0), q8.clamp(min=0)), -1)                 # [T][Hkv][g][2 D]
    R = st["max_new"]
    _, r = _rows(st)
    w = torch.zeros((st["S"], R, Hkv, g, 2 * D), device="cuda")
    w[seq, r] = both
    whole = torch.matmul(w.permute(0, 2, 3, 1, 4).reshape(st["S"], Hkv, g * R, 2 * D), b.flatten(2, 3))
    whole = whole.view(st["S"], Hkv, g, R, P).permute(0, 3, 1, 2, 4)[seq, r]                  # [T][Hkv][g][P]
    score = (whole * (sq[..., None] * st["bound_scale"][at].transpose(1, 2)[seq][:, :, None, :])).amax(2)
    i = torch.arange(P, device="cuda")
    hi = (pos // page)[:, None]
    lo = ((pos - c["window"] + 1).clamp(min=0) // page)[:, None] if c["window"] else torch.zeros_like(hi)
    ok = (i >= lo) & (i <= hi)
    kept = (i < c["first"]) | (i > hi - c["last"])
    score = score.masked_fill(kept[:, None], math.inf).masked_fill(~ok[:, None], _NINF)
    n = torch.minimum(hi - lo + 1, torch.full_like(hi, N))                   # [T][1]
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :N]
    if order.shape[-1] < N:
        order = torch.cat((order, order.new_zeros(T, Hkv, N - order.shape[-1])), -1)
    past = torch.arange(N, device="cuda") >= n[..., None]
    order = torch.where(past, torch.full_like(order, P), order).sort(-1).values
    return torch.where(past, torch.full_like(order, -1), order).int(), n.expand(T, Hkv).int().contiguous()


def _touched(st):
    """Pages that the new tokens lie on, and how many tokens each holds."""
    page = st["case"]["page"]
    q_start, kv_len = st["q_start"].long(), st["kv_len"].long()
    lo = (kv_len - (q_start[1:] - q_start[:-1])) // page
    i = torch.arange((st["max_new"] + page - 2) // page + 1, device="cuda")
    p = torch.minimum(lo[:, None] + i, ((kv_len - 1) // page)[:, None])      # (the last more than once)
    held = (kv_len[:, None] - p * page).clamp(max=page)
    return st["table"].gather(1, p).long().reshape(-1), held.reshape(-1)


def _plain_sparse(st):
    c = st["case"]
    T, Hq, Hkv, D, page, N = st["T"], c["Hq"], c["Hkv"], c["D"], c["page"], c["n_sel"]
    g = Hq // Hkv
    _plain_summarize(st, *_touched(st))
    sel, count = _plain_select(st)
    seq, pos = _positions(st)
    h = torch.arange(Hkv, device="cuda")[None, :, None]
    at = st["table"].long()[seq[:, None, None], sel.long().clamp(min=0)]     # [T][Hkv][N]
    # every page once, then each query's own
    used, back = torch.unique(at, return_inverse=True)
    kp, vp = _values_of(st, used)
    k, v = (a[back, h].reshape(T, Hkv, N * page, D) for a in (kp, vp))
    j = (sel.long()[..., None] * page + torch.arange(page, device="cuda")).view(T, Hkv, 1, N * page)
    s = torch.matmul(st["q"].float().view(T, Hkv, g, D), k.transpose(2, 3))
    del k
    if st["k_scale"] is not None:
        s *= st["k_scale"].view(1, Hkv, 1, 1)
    s, seen = _scored(st, s, pos[:, None, None, None], j, (1, Hkv, g, 1))
    s.masked_fill_(~(seen & (j >= 0)), _NINF)
    p, l, lse = _softmax(s)
    v = v * (j <= pos[:, None, None, None]).view(T, Hkv, N * page, 1)
    o = torch.matmul(p, v) / l
    if st["v_scale"] is not None:
        o *= st["v_scale"].view(1, Hkv, 1, 1)
    return (st["bounds"], st["bound_scale"], sel, count, o.reshape(T, Hq * D).to(torch.bfloat16),
            lse.reshape(T, Hq))


def run(st):
    kind = st["case"]["kind"]
    if not own:
        if kind == "tables":
            return _plain_tables(st)
        if kind == "append":
            return _plain_append(st)
        return _plain_sparse(st) if kind == "sparse" else _plain_attention(st)
    import paper_2410_06270_amd as mc
    if kind == "tables":
        mc.kv_release(st["ended"], st["past"], st["pool0"], st["batch1"], st["ws"])
        mc.kv_reserve(st["want"], st["len1"], st["pool1"], st["batch"], st["ws"], positions=st["positions"],
                      slots=st["slots"])
        return st["q_start"], st["kv_len"], st["table"], st["free"], st["n_free2"], st["positions"], st["slots"]
    if kind == "append":
        c = st["case"]
        a, b = c["Hq"] * c["D"], (c["Hq"] + c["Hkv"]) * c["D"]
        qkv = st["qkv"]
        mc.kv_append(qkv[:, :a], qkv[:, a:b], qkv[:, b:], st["prep"], st["batch"], st["cache"], st["q_out"])
        mc.kv_read(st["batch"], st["cache"], st["k_out"], st["v_out"])
        return st["q_out"], st["k_out"], st["v_out"]
    if kind == "sparse":
        c = st["case"]
        mc.kv_summarize(st["batch"], st["cache"], st["summary"])
        mc.attn_select(st["q"], st["batch"], st["cache"], st["summary"], st["attn"], st["sel"], st["count"], st["ws"],
                       keep_first=c["first"], keep_last=c["last"])
        mc.attn_sparse(st["q"], st["batch"], st["cache"], st["attn"], st["sel"], st["count"], st["o"], st["ws"],
                       lse=st["lse"])
        return st["bounds"], st["bound_scale"], st["sel"], st["count"], st["o"], st["lse"]
    attend = mc.attn_decode if kind == "decode" else mc.attn_prefill
    attend(st["q"], st["batch"], st["cache"], st["attn"], st["o"], st["ws"], lse=st["lse"])
    return st["o"], st["lse"]


# -------------------------------------------------------------------- work --

def _element_bytes(case):
    return {"bf16": 2.0, "e4m3": 1.0, "e2m1": 17 / 32}[case["kv"]]


def _visible(case, new, past):
    """Visible (row, key) pairs of a sequence, and the keys that some row sees."""
    w, f = case["window"], min(case["prefix"], past + new)
    first = max(0, past - w + 1) if w else 0
    keys = past + new - first + min(f, first)
    lo = torch.arange(past, past + new, dtype=torch.float64)
    start = torch.clamp(lo - w + 1, min=0) if w else torch.zeros_like(lo)
    more = torch.minimum(start, torch.full_like(lo, f)) + torch.clamp(f - 1 - lo, min=0)
    return float((lo - start + 1 + more).sum()), keys


def work(case):
    n = _lengths(case)
    T, S = sum(a for a, _ in n), len(n)
    if case["kind"] == "tables":
        page = case["page"]
        moved = sum(-(-(a + b) // page) - -(-b // page) for a, b in n)
        return {"bytes": S * 17 + moved * 8 + T * 12, "flops": T + 10 * S}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    e = _element_bytes(case)
    if case["kind"] == "append":
        # read and written, and the new tokens read back
        return {"bytes": T * D * (2 * (2 * Hq + 2 * Hkv) + 2 * e * Hkv + (2 * e + 4) * Hkv) + T * case["rot"] * 4,
                "flops": T * D * ((Hq + Hkv) * (3 + (4 if case["norm"] != "none" else 0)) + 8 * Hkv)}
    if case["kind"] == "sparse":
        page, N, w = case["page"], case["n_sel"], case["window"]
        byts, flops = 0.0, 0.0
        for a, b in n:
            pages = (a + b - 1) // page + 1
            byts += pages * Hkv * (2 * D + 4)
            # pages that only some rows take are read for them; no sequence has to read more than it has
            keys = min(a * N * page, a + b)
            byts += keys * Hkv * D * 2 * e + (a + page) * Hkv * D * e
            rows = torch.arange(b, a + b, dtype=torch.float64)
            flops += 4.0 * Hq * D * float(torch.clamp(rows + 1, max=min(N * page, w or N * page)).sum())
            flops += 2.0 * Hq * D * float((rows // page + 1).sum())
        return {"bytes": byts + T * Hq * (4 * D + 4) + T * Hkv * 4 * (N + 1), "flops": flops}
    seen = [_visible(case, a, b) for a, b in n]
    pairs, keys = sum(p for p, _ in seen), sum(k for _, k in seen)
    return {"bytes": keys * Hkv * D * 2 * e + T * Hq * (4 * D + 4), "flops": 4.0 * Hq * D * pairs}


# ------------------------------------------------------------------- exact --

def _head64(st, s, h, n):
    """Keys and values 0 .. n-1 of sequence s and head h in 64 bits, by the
    byte addresses of the layout."""
    c = st["case"]
    D, page, Hkv = c["D"], c["page"], c["Hkv"]
    t = torch.arange(n, device="cuda")
    d = torch.arange(D, device="cuda")[None]
    pg = st["table"][s].long()[t // page][:, None]
    blk = h * (page // 16) + (t % page)[:, None] // 16
    i = (t % 16)[:, None]
    k, v = (st[a].view(torch.uint8) for a in ("k_cache", "v_cache"))
    if c["kv"] == "e2m1":
        cut = Hkv * page * D // 2
        table = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device="cuda") / 2

        def value(code):
            return table[(code & 7).long()] * (1 - 2 * (code >> 3).double())

        kb = k[pg, blk * 8 * D + d // 32 * 256 + i * 16 + d % 32 // 2]
        vb = v[pg, blk * 8 * D + d // 32 * 256 + d % 16 * 16 + d // 16 % 2 * 8 + i // 2]
        kx = k[pg, cut + blk * (D // 2) + d // 32 * 16 + i % 4 * 4 + i // 4].double()
        vx = v.view(torch.bfloat16)[pg, cut // 2 + blk * (D // 4) + d // 64 * 16 + i].double()
        return value(kb >> (d % 2 * 4) & 15) * torch.exp2(kx - 127), value(vb >> (i % 2 * 4) & 15) * vx
    U = 16 // st["k_cache"].element_size()
    kt = st["k_cache"].dtype
    raw = torch.uint8 if U == 16 else torch.int16
    ak = blk * 16 * D + d // U * 16 * U + i * U + d % U
    av = blk * 16 * D + i // U * D * U + d * U + i % U
    k, v = (a.view(raw)[pg, at].view(kt).double() for a, at in ((k, ak), (v, av)))
    if st["k_scale"] is not None:
        k, v = k * st["k_scale"][h].double(), v * st["v_scale"][h].double()
    return k, v


def _exact_scores(st, q, k, hq, i, j):
    c = st["case"]
    z = (q @ k.t()) * st["scale"]
    if c["cap"]:
        z = c["cap"] * torch.tanh(z / c["cap"])
    if st["slopes"] is not None:
        z = z + st["slopes"][hq].double() * (j - i)
    ok = (j <= i) & ((j > i - c["window"]) if c["window"] else (j >= 0))
    if c["prefix"]:
        ok = ok | (j < c["prefix"])
    return z, ok


def exact(case, seed):
    global own
    if case["kind"] == "tables":      # whole numbers throughout
        return None
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    n = _lengths(case)
    if case["kind"] == "append":
        return _exact_append(st, n)
    Hq, Hkv, D, page = case["Hq"], case["Hkv"], case["D"], case["page"]
    o = torch.zeros((st["T"], Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((st["T"], Hq), dtype=torch.float64, device="cuda")
    sel = None
    if case["kind"] == "sparse":
        _plain_summarize(st, *_touched(st))
        sel = _plain_select(st)[0].long()
    q0 = 0
    for s, (a, b) in enumerate(n):
        i = torch.arange(b, a + b, device="cuda")[:, None]
        j = torch.arange(a + b, device="cuda")[None]
        for h in range(Hkv):
            k, v = _head64(st, s, h, a + b)
            taken = None
            if sel is not None:
                taken = torch.zeros((a, (a + b - 1) // page + 2), dtype=torch.bool, device="cuda")
                mine = sel[q0:q0 + a, h]
                taken.scatter_(1, torch.where(mine < 0, torch.full_like(mine, taken.shape[1] - 1), mine), True)
                taken = taken[:, (j // page)[0]]
            for hq in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                z, ok = _exact_scores(st, st["q"][q0:q0 + a, hq * D:(hq + 1) * D].double(), k, hq, i, j)
                z = torch.where(ok if taken is None else ok & taken, z, torch.full_like(z, _NINF))
                w = torch.logsumexp(z, 1)
                lse[q0:q0 + a, hq] = w
                o[q0:q0 + a, hq] = torch.exp(z - w[:, None]) @ v
        q0 += a
    o = o.view(st["T"], Hq * D)
    return (o, lse) if sel is None else (None, None, None, None, o, lse)


def _exact_append(st, n):
    """Queries, keys and values after norm and rotation; keys and values as the levels of
    their groups that lie nearest."""
    c = st["case"]
    Hq, Hkv, D, rot = c["Hq"], c["Hkv"], c["D"], c["rot"]
    x = st["qkv"].double()
    levels = torch.tensor(_LEVELS, dtype=torch.float64, device="cuda")
    mids = (levels[1:] + levels[:-1]) / 2

    def level(a):                     # the even code of two as near: a border belongs to it
        up = torch.bucketize(a, mids, right=True)
        down = torch.bucketize(a, mids)
        return levels[torch.where(up % 2 == 0, up, down)]

    out = []
    pos = torch.cat([torch.arange(b, a + b, device="cuda") for a, b in n])
    for first, heads, w, kind in ((0, Hq, st["q_norm"], "q"), (Hq, Hkv, st["k_norm"], "k"), (Hq + Hkv, Hkv, None, "v")):
        y = x[:, first * D:(first + heads) * D]
        if w is not None and c["norm"] == "row":
            y = y * w.double() * (y.pow(2).sum(1, keepdim=True) / (heads * D) + _EPS).pow(-0.5)
        y = y.reshape(-1, heads, D)
        if w is not None and c["norm"] == "head":
            y = y * w.double() * (y.pow(2).sum(2, keepdim=True) / D + _EPS).pow(-0.5)
        if rot and kind != "v":
            i = torch.arange(rot // 2, device="cuda")
            lo, hi = (2 * i, 2 * i + 1) if c["pairs"] else (i, i + rot // 2)
            z = torch.complex(y[..., lo], y[..., hi])
            z = z * torch.complex(st["rope"][pos, :, 0].double(), st["rope"][pos, :, 1].double())[:, None]
            y = y.clone()
            y[..., lo], y[..., hi] = z.real, z.imag
        if kind == "k":
            b = y.reshape(-1, heads, D // 32, 32)
            unit = torch.exp2(torch.ceil(torch.log2(b.abs().amax(-1, keepdim=True) / 7)))
            y = level((b / unit).abs()) * torch.sign(b) * unit
        elif kind == "v":
            b = y.reshape(-1, heads, D // 64, 64)
            s = (b.abs().amax(-1, keepdim=True).float() / 6).double()
            m, e = torch.frexp(s)
            s = torch.ldexp((m * 64).round() / 64, e)
            y = level((b / s).abs()) * torch.sign(b) * s
        out.append(y.reshape(-1, heads * D))
    return tuple(out)
