"""Caps, scales and scores over the whole range that the attention calls take, against
the 64-bit oracle."""
import math

import pytest

torch = pytest.importorskip("torch")

from oracle import attention as oa  # noqa: E402
from test_gpu_attention import BF16, E4M3, World, mc, run_attention, starts  # noqa: E402,F401

pytestmark = pytest.mark.gpu

CAPS = [65.0, 1e3, 1e5, 1e8, 1e30, 2.0 ** 126]


@pytest.mark.parametrize("cap", [0.5, 64.0] + CAPS)
@pytest.mark.parametrize("which", ["decode", "prefill"])
def test_capped_score_of_one_key(mc, cap, which):
    """With one key lse is the capped score itself.  Products of two bf16 values
    are exact; from 2^-24 to 1.9 of the cap either way, and some ordinary ones."""
    S, Hq, D, page = 64, 16, 64, 16
    gen = torch.Generator().manual_seed(21)
    b = torch.exp2(torch.linspace(-24.0, math.log2(1.9), S)) * (cap if cap < 1e30 else 2.0 ** 26)
    b[1::7] = torch.tensor([0.3, 1.0, 3.0, -2.0, 20.0] * 2)[:b[1::7].numel()]
    b[::2] = -b[::2]
    b = b.to(BF16)
    a = (0.5 + 0.5 * torch.rand(Hq, generator=gen)).to(BF16)
    far = 1.0 if cap < 1e30 else 2.0 ** math.floor(math.log2(cap) - 26)      # the rest of a far cap, exact
    q = torch.zeros((S, Hq, D), dtype=BF16)
    q[:, :, 3] = a * far
    q[1::7, :, 3] = a                                            # the ordinary ones
    k = torch.zeros((S, page, D), dtype=BF16)
    k[:, 0, 3] = b
    flat = torch.zeros((S * page * D,), dtype=BF16)
    table = torch.arange(S, dtype=torch.int32).view(S, 1)
    for s in range(S):
        oa.write("k", flat, table[s], torch.arange(1), 0, k[s, :1], page, 1, D, 8)
    cache = mc.KVCache(S, page, 1, D, k=flat.view(S, -1).cuda(), v=torch.ones((S, page * D), dtype=BF16, device="cuda"))
    kw = {} if which == "decode" else dict(q_start=starts([1] * S), T=S)
    batch = mc.KVBatch(torch.ones(S, dtype=torch.int32, device="cuda"), table.cuda(), **kw)
    o, lse = torch.empty((S, Hq * D), dtype=BF16, device="cuda"), torch.empty((S, Hq), device="cuda")
    ws = torch.empty(mc.attn_workspace(S, Hq, 1, D), dtype=torch.uint8, device="cuda")
    call = mc.attn_decode if which == "decode" else mc.attn_prefill
    call(q.view(S, -1).cuda(), batch, cache, mc.Attention(Hq, 1.0, softcap=cap), o, ws, lse=lse)
    torch.cuda.synchronize()
    x = q[:, :, 3].double() * b.double()[:, None]
    cap = float(torch.tensor(cap, dtype=torch.float32))
    want = cap * torch.tanh(x / cap)
    # the cap's own error as the oracle has it, and six roundings between the
    # domains of the two logarithms
    tol = oa.cap_error(want, cap) + 6 * oa.U24 * want.abs()
    off = (lse.cpu().double() - want).abs()
    assert bool((off <= tol).all()), "%g of its bound" % float((off / tol).max())
    assert bool((o == 1).all())


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("D,dtype,slopes", [(64, BF16, False), (128, BF16, True), (64, E4M3, True), (128, E4M3, False)])
def test_large_caps(mc, cap, D, dtype, slopes):
    """Decode, prefill (one team and two) and importance with caps that hardly bind."""
    sl = torch.exp2(-torch.arange(1, 5, dtype=torch.float32)) if slopes else None
    w = World(mc, [1, 77, 300], Hkv=2, D=D, page=32, dtype=dtype, seed=D)
    kw = dict(cap=cap, slopes=sl)
    run_attention(mc, w, None, 4, True, what="decode, large cap", **kw)
    for max_len in (0, 512):
        run_attention(mc, w, [1, 30, 300], 4, False, max_len=max_len, what="prefill, large cap", **kw)
    L = 200
    w = World(mc, [L], Hkv=2, D=D, page=32, dtype=dtype, seed=D + 1)
    q = w.randn(L + 3, 4 * D).to(BF16)
    _, lse = run_attention(mc, w, [L], 4, False, q=q, what="importance, large cap", **kw)
    lse = lse[:L].contiguous()
    x = w.randn(L, 64).to(BF16)
    batch = mc.KVBatch(torch.tensor([L], dtype=torch.int32, device="cuda"), w.table.cuda(), q_start=starts([L]), T=L)
    imp, mask = torch.empty(L, device="cuda"), torch.empty(L, dtype=torch.uint8, device="cuda")
    ws = torch.empty(mc.attn_importance_workspace(4, L), dtype=torch.uint8, device="cuda")
    at = mc.Attention(4, D ** -0.5, softcap=cap, slopes=None if sl is None else sl.cuda())
    mc.attn_importance(q[:L].cuda(), lse, batch, w.cache, at, x.cuda(), 0.1, mask, ws, importance=imp)
    torch.cuda.synchronize()
    want, rel = oa.importance(q[:L].double(), lse.double().cpu(), [w.rows("k", 0, h) for h in range(2)], x.double(), L,
                              2, 2, D, scale=D ** -0.5, cap=cap, slopes=sl)
    assert bool(((imp.cpu().double() - want).abs() <= rel * want).all())


@pytest.mark.parametrize("scale", [2.0 ** 126, -2.0 ** 126, 2.0 ** -126])
@pytest.mark.parametrize("which", ["decode", "prefill"])
def test_scales_at_the_limit(mc, scale, which):
    """One key and products of 2^-scale's exponent: lse is the score, an ordinary one."""
    Hq, D, page = 4, 64, 16
    k = torch.zeros((1, D), dtype=BF16)
    k[0, 5] = math.copysign(math.ldexp(1.25, -63 if abs(scale) > 1 else 63), scale)
    flat = torch.zeros((page * D,), dtype=BF16)
    table = torch.zeros((1, 1), dtype=torch.int32)
    oa.write("k", flat, table[0], torch.arange(1), 0, k, page, 1, D, 8)
    q = torch.zeros((1, Hq, D), dtype=BF16)
    q[0, :, 5] = torch.tensor([1.0, 1.5, -1.75, 0.0]) * 2.0 ** (-61 if abs(scale) > 1 else 63)
    cache = mc.KVCache(1, page, 1, D, k=flat.view(1, -1).cuda(), v=torch.ones((1, page * D), dtype=BF16, device="cuda"))
    kw = {} if which == "decode" else dict(q_start=starts([1]), T=1)
    batch = mc.KVBatch(torch.ones(1, dtype=torch.int32, device="cuda"), table.cuda(), **kw)
    o, lse = torch.empty((1, Hq * D), dtype=BF16, device="cuda"), torch.empty((1, Hq), device="cuda")
    ws = torch.empty(mc.attn_workspace(1, Hq, 1, D), dtype=torch.uint8, device="cuda")
    call = mc.attn_decode if which == "decode" else mc.attn_prefill
    call(q.view(1, -1).cuda(), batch, cache, mc.Attention(Hq, scale), o, ws, lse=lse)
    torch.cuda.synchronize()
    want = q[0, :, 5].double() * k[0, 5].double() * scale
    # log2(e), the scale and the score in the log2 domain, ln 2 and lse rounded
    assert bool(((lse[0].cpu().double() - want).abs() <= 6 * oa.U24 * want.abs()).all())
    assert bool((o == 1).all())


def _far_scores(mc, D, dtype, e, scale, Hq=2, L=1100, seed=22):
    """A world of one sequence whose scores are scale 2^e times one dimension of the keys,
    queries for it and the scores in units of 2^e (and of an e4m3 head's scale)."""
    gen = torch.Generator().manual_seed(seed)
    e4 = dtype == E4M3
    steps = torch.arange(0x20, 0x78, dtype=torch.uint8) if e4 else torch.arange(0x3f80, 0x3f80 + 1200, dtype=torch.int16)
    if e4:
        kv = steps.view(E4M3)[torch.randint(len(steps), (L,), generator=gen)].double()
    else:
        kv = steps.view(BF16)[torch.randperm(len(steps), generator=gen)[:L]].double()
    odd = [(0, slice(None), 0, 0, "k", kv.float().to(dtype))]
    w = World(mc, [L], Hkv=1, D=D, page=64, dtype=dtype, seed=seed, odd=odd)
    q = torch.zeros((L, Hq * D), dtype=BF16)
    q[:, ::D] = 2.0 ** e
    return w, q, kv if scale > 0 else -kv


def _best(kv, v, pos):
    """The mean of the values at the largest score that each position sees."""
    rows = []
    for i in pos.tolist():
        seen = kv[:i + 1]
        rows.append(v[:i + 1][seen == seen.max()].mean(0))
    return torch.stack(rows)


@pytest.mark.parametrize("e", [20, 27, 31, 33, 40, 100])
@pytest.mark.parametrize("D,dtype", [(64, BF16), (128, BF16), (64, E4M3), (128, E4M3)])
@pytest.mark.parametrize("sign", [1, -1])
def test_far_scores(mc, e, D, dtype, sign):
    """Finite scores of any size choose the keys that have the largest: prefill in one
    part, two teams and several parts, and decode."""
    Hq, L, new = 2, 1100, 400
    w, q, kv = _far_scores(mc, D, dtype, e, sign)
    v = w.rows("v", 0, 0)
    pos = torch.arange(L - new, L)
    want = _best(kv, v, pos)
    top = torch.stack([kv[:i + 1].max() for i in pos.tolist()])
    if w.scale["k"] is not None:
        top = top * w.scale["k"][0].double()
    top = top * 2.0 ** e
    # the weights' rounding and the output's; gaps are 160 or more
    tol = 2 * oa.BF * v.abs().amax()
    # ln of up to 1100 ties, and the roundings of a score in two domains and the head's scale
    tol_l = 8 * oa.U24 * top.abs() + 8
    n = torch.tensor([L], dtype=torch.int32, device="cuda")
    for what, max_len in (("decode", 0), ("decode", 1), ("prefill", 1), ("prefill", 512), ("prefill", 0)):
        rows = 1 if what == "decode" else new
        kw = {} if what == "decode" else dict(q_start=starts([new]), T=new)
        batch = mc.KVBatch(n, w.table.cuda(), max_len=max_len, **kw)
        o, lse = torch.empty((rows, Hq * D), dtype=BF16, device="cuda"), torch.empty((rows, Hq), device="cuda")
        call = mc.attn_decode if what == "decode" else mc.attn_prefill
        call(q[-rows:].cuda(), batch, w.cache, mc.Attention(Hq, float(sign)), o, w.workspace(mc, rows, Hq), lse=lse)
        torch.cuda.synchronize()
        for h in range(Hq):
            off = (o[:, h * D:(h + 1) * D].cpu().double() - want[-rows:]).abs()
            assert bool((off <= tol).all()), (what, max_len, h)
            assert bool(((lse[:, h].cpu().double() - top[-rows:]).abs() <= tol_l[-rows:]).all()), (what, max_len, h)


@pytest.mark.parametrize("D,max_len", [(64, 1), (64, 512), (64, 0), (128, 1), (128, 0)])
@pytest.mark.parametrize("prefix", [None, 900])
@pytest.mark.parametrize("first", [2.0 ** -40, 0.0, -1.0])
def test_scores_that_become_far(mc, D, max_len, prefix, first):
    """Ordinary scores, zeros or far negative ones in the first tiles, far ones behind them."""
    Hq, L, new, cut = 2, 1100, 400, 777
    w, q, kv = _far_scores(mc, D, BF16, 40, 1)
    k = torch.zeros((cut, D), dtype=BF16)
    k[:, 0] = (kv[:cut] * first).float().to(BF16)
    kv[:cut] = k[:, 0].double()
    flat = w.flat["k"].clone()
    was = w.rows("k", 0, 0)[:cut].to(BF16)
    was[:, 0] = k[:, 0]
    oa.write("k", flat, w.table[0], torch.arange(cut), 0, was, w.page, 1, D, 8)
    w.cache.k.copy_(flat.view(w.cache.k.shape))
    v = w.rows("v", 0, 0)
    pos = torch.arange(L - new, L)
    s = kv * 2.0 ** 40
    want = torch.stack([torch.softmax(s[:max(i + 1, prefix or 0)], 0) @ v[:max(i + 1, prefix or 0)] for i in pos.tolist()])
    # in rows before the far scores the weights' rounding, the sums of 1100 terms, and twice the
    # roundings of scores up to 4
    tol = (2 * oa.BF + (2 * L + 64) * oa.U24) * v.abs().amax()
    batch = mc.KVBatch(torch.tensor([L], dtype=torch.int32, device="cuda"), w.table.cuda(), q_start=starts([new]), T=new,
                       max_len=max_len)
    at = mc.Attention(Hq, 1.0, prefix=None if prefix is None else torch.tensor([prefix], dtype=torch.int32, device="cuda"))
    o = torch.empty((new, Hq * D), dtype=BF16, device="cuda")
    mc.attn_prefill(q[-new:].cuda(), batch, w.cache, at, o, w.workspace(mc, new, Hq))
    torch.cuda.synchronize()
    for h in range(Hq):
        assert bool(((o[:, h * D:(h + 1) * D].cpu().double() - want).abs() <= tol).all()), h
