"""Caps and scales over the whole range that the attention calls take, against the
64-bit oracle."""
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
