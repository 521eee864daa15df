"""Capped scores of rows that see few keys, whatever the size of the call they are in, its hint of the lengths and
the kind of cache: in decode and over selected pages each score is off by a few roundings of itself, not of the
cap; in prefill so above a cap of 64, and up to it by those of the cap.

A query has one element, so its product with a key is exact in fp32, and a row that sees one key has as its lse that
key's capped score alone: its weight, sum and logarithm are 1, 1 and 0 exactly."""
import math

import pytest

torch = pytest.importorskip("torch")

import test_gpu_attention as ta  # noqa: E402
import test_gpu_sparse as ts  # noqa: E402
from oracle import attention as oa  # noqa: E402

pytestmark = pytest.mark.gpu

mc = ta.mc
BF16, E4M3, E2M1 = ts.BF16, ts.E4M3, ts.E2M1
U24 = oa.U24
LENS = [300, 1, 45, 20, 0, 700]
HQ, HKV = 4, 2

# Half steps of fp32 relative to the score: 28 of the capped score (oracle.attention.cap_error, its relative form),
# 12 of its factors: the call's scale, the cache's, their product with log2 e, the quotient by the cap and
# twice that with log2 e (two roundings each), the product with ln 2 at the end.
SCORE = 40


def queries(w, rows):
    """Rows [rows][HQ * D] whose heads have one element each."""
    q = torch.zeros((rows, HQ, w.D))
    at = torch.randint(0, w.D, (rows, HQ), generator=w.gen)
    q.scatter_(2, at[..., None], w.randn(rows, HQ, 1))
    return q.to(BF16).view(rows, HQ * w.D)


def capped(w, q, row, s, j, hq, cap, scale):
    """The capped score of query row `row` and key j of sequence s."""
    held = w.__dict__.setdefault("held", {})
    at = s, hq * HKV // HQ
    if at not in held:
        held[at] = w.rows("k", *at, LENS[s])
    z = float(q[row, hq * w.D:(hq + 1) * w.D].double() @ held[at][j]) * scale
    return cap * math.tanh(z / cap)


def check_one(got, want, what, cap=None):
    """cap: where errors are the cap's (oracle.attention.cap_error, whose 28 half steps of the score SCORE holds)."""
    room = SCORE * U24 * abs(want) + (8 * U24 * cap if cap is not None and cap <= 64 else 0.0)
    assert abs(float(got) - want) <= room, "%s: %.9g for %.9g" % (what, float(got), want)


def world(mc, kind, D, page=16):
    return ts.world(mc, kind, LENS, Hkv=HKV, D=D, page=page, seed=D + page, gap=2)


@pytest.mark.parametrize("kind", [BF16, E4M3, E2M1])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [0.3, 20.0, 50.0, 64.0, 100.0])
def test_prefill(mc, kind, D, cap):
    """First tokens of long and short prompts, and rows that a window of one leaves themselves."""
    w = world(mc, kind, D)
    T, scale = sum(LENS), D ** -0.5
    q = queries(w, T)
    batch = lambda hint: mc.KVBatch(torch.tensor(LENS, dtype=torch.int32, device="cuda"), w.table.cuda(),  # noqa: E731
                                    q_start=ta.starts(LENS), T=T, max_len=hint)
    for window in (0, 1):
        first = None
        for hint in (0, 16, 300):
            o = torch.zeros((T, HQ * D), dtype=BF16, device="cuda")
            lse = torch.zeros((T, HQ), device="cuda")
            print("prefill", kind, D, cap, window, hint, flush=True)
            mc.attn_prefill(q.cuda(), batch(hint), w.cache, mc.Attention(HQ, scale, softcap=cap, window=window), o,
                            w.workspace(mc, T, HQ), lse=lse)
            torch.cuda.synchronize()
            got, row = lse.cpu(), 0
            alone = []
            for s, n in enumerate(LENS):
                for j in range(n if window else min(n, 1)):
                    for hq in range(HQ):
                        check_one(got[row + j, hq], capped(w, q, row + j, s, j, hq, cap, scale), "s=%d j=%d" % (s, j), cap)
                    alone.append(row + j)
                row += n
            if first is None:
                first = got[alone]
            assert torch.equal(got[alone], first)            # the hint changes nothing where nothing is summed


@pytest.mark.parametrize("kind", [BF16, E4M3, E2M1])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [0.3, 20.0, 50.0, 64.0, 100.0])
def test_decode(mc, kind, D, cap):
    """A sequence of one token beside long ones, and windows of one."""
    w = world(mc, kind, D)
    S, scale = len(LENS), D ** -0.5
    q = queries(w, S)
    for window in (0, 1):
        first = None
        for hint in (0, 16, 300):
            batch = mc.KVBatch(torch.tensor(LENS, dtype=torch.int32, device="cuda"), w.table.cuda(), max_len=hint)
            o = torch.zeros((S, HQ * D), dtype=BF16, device="cuda")
            lse = torch.zeros((S, HQ), device="cuda")
            print("decode", kind, D, cap, window, hint, flush=True)
            mc.attn_decode(q.cuda(), batch, w.cache, mc.Attention(HQ, scale, softcap=cap, window=window), o,
                           w.workspace(mc, S, HQ), lse=lse)
            torch.cuda.synchronize()
            got = lse.cpu()
            alone = [s for s, n in enumerate(LENS) if n == 1 or (window and n)]
            for s in alone:
                for hq in range(HQ):
                    check_one(got[s, hq], capped(w, q, s, s, LENS[s] - 1, hq, cap, scale), "s=%d" % s)
            if first is None:
                first = got[alone]
            assert torch.equal(got[alone], first)


@pytest.mark.parametrize("kind", [BF16, E4M3, E2M1])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize("n_sel", [4, 80])
@pytest.mark.parametrize("cap", [20.0, 50.0, 64.0, 100.0])
def test_sparse(mc, kind, D, page, n_sel, cap):
    """Rows at their sequence's first place, and rows with a window of one, of short and long lists."""
    w = world(mc, kind, D, page)
    new = [min(n, 40) for n in LENS]
    T, scale, P = sum(new), D ** -0.5, w.table.shape[1]
    q = queries(w, T)
    pos = [(s, n - m + i) for s, (n, m) in enumerate(zip(LENS, new)) for i in range(m)]
    sel = torch.full((T, HKV, n_sel), -1, dtype=torch.int32)
    count = torch.zeros((T, HKV), dtype=torch.int32)
    for t, (s, j) in enumerate(pos):
        m = min(n_sel, j // page + 1)
        sel[t, :, :m] = torch.arange(j // page - m + 1, j // page + 1, dtype=torch.int32)
        count[t] = m
    batch = mc.KVBatch(torch.tensor(LENS, dtype=torch.int32, device="cuda"), w.table.cuda(), q_start=ta.starts(new), T=T)
    for window in (0, 1):
        o = torch.zeros((T, HQ * D), dtype=BF16, device="cuda")
        lse = torch.zeros((T, HQ), device="cuda")
        print("sparse", kind, D, page, n_sel, cap, window, flush=True)
        mc.attn_sparse(q.cuda(), batch, w.cache, mc.Attention(HQ, scale, softcap=cap, window=window), sel.cuda(),
                       count.cuda(), o, w.workspace(mc, T, HQ), lse=lse)
        torch.cuda.synchronize()
        got = lse.cpu()
        for t, (s, j) in enumerate(pos):
            if j == 0 or window:
                for hq in range(HQ):
                    check_one(got[t, hq], capped(w, q, t, s, j, hq, cap, scale), "s=%d j=%d" % (s, j))


@pytest.mark.parametrize("kind", [BF16, E4M3, E2M1])
@pytest.mark.parametrize("kw", [dict(), dict(window=9), dict(window=33, prefix=[5, 1, 40, 20, 0, 70]),
                                dict(slopes=True), dict(window=20, slopes=True, prefix=[0, 1, 2, 0, 0, 30])])
def test_few_keys_among_many(mc, kind, kw):
    """Rows of one to some hundred keys, random queries: o and lse within the oracle's bounds."""
    w = world(mc, kind, 128)
    if kw.get("slopes"):
        kw = dict(kw, slopes=torch.exp2(-torch.arange(1, HQ + 1).float()))
    for cap in (0.01, 50.0):
        ta.run_attention(mc, w, LENS, HQ, False, cap=cap, what="few", **kw)
        ta.run_attention(mc, w, None, HQ, True, cap=cap, what="few", **kw)
