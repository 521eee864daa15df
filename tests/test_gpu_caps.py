"""Capped scores of rows that see few keys, whatever the size of the call they are in, its hint of the lengths and
the kind of cache: each score is off by a few roundings of itself, not of the cap.

A query has one element, so its product with a key is exact in fp32.  A row that sees one key has as its lse that key's
capped score alone: its weight, sum and logarithm are 1, 1 and 0 exactly."""
import pytest

torch = pytest.importorskip("torch")

import test_gpu_attention as ta  # noqa: E402
import test_gpu_sparse as ts  # noqa: E402
from oracle import attention as oa  # noqa: E402

pytestmark = pytest.mark.gpu

mc = ta.mc
BF16, E4M3, E2M1 = ts.BF16, ts.E4M3, ts.E2M1
U24 = oa.U24
LENS = [300, 1, 45, 20, 0, 31, 2, 700]
HQ, HKV = 4, 2

# Half steps of fp32 relative to the score: 28 of the capped score (oracle.attention.cap_error, its relative form),
# 12 of its factors: the call's scale, the cache's, their product with log2 e, the quotient by the cap and
# twice that with log2 e (two roundings each), the product with ln 2 at the end.
SCORE = 40
# Rows of fewer keys than these have them (in prefill, at the first positions).
PREFILL, DECODE = 8, 32


def queries(w, rows):
    """Rows [rows][HQ * D] whose heads have one element each."""
    q = torch.zeros((rows, HQ, w.D))
    at = torch.randint(0, w.D, (rows, HQ), generator=w.gen)
    q.scatter_(2, at[..., None], w.randn(rows, HQ, 1))
    return q.to(BF16).view(rows, HQ * w.D)


def check_rows(w, q, got, rows, cap, scale, window, few, prefix=None):
    """rows: (row of q and got, sequence, position).  Checks those that see fewer than `few` keys; returns rows of one.

    The lse of n keys: the scores' errors at most; of each weight a step of exp2, which is two half steps, and one of
    its argument, n additions, a step of log2, near 1 of 1: n + 7; 4 half steps of the lse itself (sum, product, ln 2)."""
    held, alone, most = {}, [], 0
    for t, s, j in rows:
        keys = set(range(max(0, j - window + 1) if window else 0, j + 1))
        keys = sorted(keys | set(range(min(prefix[s], LENS[s]) if prefix else 0)))
        n = len(keys)
        if n >= few:
            continue
        most = max(most, n)
        for hq in range(HQ):
            at = s, hq * HKV // HQ
            if at not in held:
                held[at] = w.rows("k", *at, LENS[s])
            z = (held[at][keys] @ q[t, hq * w.D:(hq + 1) * w.D].double()) * scale
            z = cap * torch.tanh(z / cap)
            want, top = float(torch.logsumexp(z, 0)), float(z.abs().max())
            room = SCORE * U24 * top + (0.0 if n == 1 else (n + 7) * U24 + 4 * U24 * abs(want))
            off = abs(float(got[t, hq]) - want)
            assert off <= room, "s=%d j=%d keys=%d: %.9g for %.9g" % (s, j, n, got[t, hq], want)
        if n == 1:
            alone.append(t)
    assert most == min(few - 1, window or few - 1) or prefix
    return alone


def world(mc, kind, D, page=16):
    return ts.world(mc, kind, LENS, Hkv=HKV, D=D, page=page, seed=D + page, gap=2)


CASES = dict(argnames="cap", argvalues=[0.3, 20.0, 50.0, 64.0, 100.0])


@pytest.mark.parametrize("kind", [BF16, E4M3, E2M1])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize(**CASES)
def test_prefill(mc, kind, D, page, cap):
    """First tokens of long and short prompts, in parts and teams or not, with windows and prefixes."""
    w = world(mc, kind, D, page)
    T, scale = sum(LENS), -D ** -0.5 if cap == 20.0 else D ** -0.5
    q = queries(w, T)
    rows = [(t, s, j) for t, (s, j) in enumerate((s, j) for s, n in enumerate(LENS) for j in range(n))
            if j < PREFILL - 1]
    for window, prefix in ((0, None), (1, None), (3, None), (40, None), (0, [5, 1, 7, 70, 0, 3, 2, 6]),
                           (2, [5, 1, 7, 70, 0, 3, 2, 6])):
        pre = None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device="cuda")
        first = None
        for hint in (0, 16, 300, 2000):
            batch = mc.KVBatch(torch.tensor(LENS, dtype=torch.int32, device="cuda"), w.table.cuda(),
                               q_start=ta.starts(LENS), T=T, max_len=hint)
            o = torch.zeros((T, HQ * D), dtype=BF16, device="cuda")
            lse = torch.zeros((T, HQ), device="cuda")
            print("prefill", kind, D, cap, window, hint, flush=True)
            at = mc.Attention(HQ, scale, softcap=cap, window=window, prefix=pre)
            mc.attn_prefill(q.cuda(), batch, w.cache, at, o, w.workspace(mc, T, HQ), lse=lse)
            torch.cuda.synchronize()
            got = lse.cpu()
            alone = check_rows(w, q, got, rows, cap, scale, window, PREFILL, prefix)
            first = got[alone] if first is None else first
            assert torch.equal(got[alone], first)            # the hint changes nothing where nothing is summed


@pytest.mark.parametrize("kind", [BF16, E4M3, E2M1])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize(**CASES)
def test_decode(mc, kind, D, page, cap):
    """Short sequences beside long ones, and windows of few keys."""
    w = world(mc, kind, D, page)
    S, scale = len(LENS), D ** -0.5
    q = queries(w, S)
    rows = [(s, s, n - 1) for s, n in enumerate(LENS) if n]
    for window, prefix in ((0, None), (1, None), (9, None), (31, None), (3, [5, 1, 27, 20, 0, 3, 2, 28])):
        pre = None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device="cuda")
        first = None
        for hint in (0, 16, 300):
            batch = mc.KVBatch(torch.tensor(LENS, dtype=torch.int32, device="cuda"), w.table.cuda(), max_len=hint)
            o = torch.zeros((S, HQ * D), dtype=BF16, device="cuda")
            lse = torch.zeros((S, HQ), device="cuda")
            print("decode", kind, D, cap, window, hint, flush=True)
            mc.attn_decode(q.cuda(), batch, w.cache, mc.Attention(HQ, scale, softcap=cap, window=window, prefix=pre), o,
                           w.workspace(mc, S, HQ), lse=lse)
            torch.cuda.synchronize()
            got = lse.cpu()
            alone = check_rows(w, q, got, rows, cap, scale, window, DECODE, prefix)
            first = got[alone] if first is None else first
            assert torch.equal(got[alone], first)


@pytest.mark.parametrize("kind", [BF16, E4M3, E2M1])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize("n_sel", [4, 80])
@pytest.mark.parametrize(**CASES)
def test_sparse(mc, kind, D, page, n_sel, cap):
    """Rows at their sequence's first places, and rows with windows of few keys, of short and long lists."""
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
    batch = mc.KVBatch(torch.tensor(LENS, dtype=torch.int32, device="cuda"), w.table.cuda(), q_start=ta.starts(new),
                       T=T)
    for window in (0, 1, 9, 31):
        o = torch.zeros((T, HQ * D), dtype=BF16, device="cuda")
        lse = torch.zeros((T, HQ), device="cuda")
        print("sparse", kind, D, page, n_sel, cap, window, flush=True)
        mc.attn_sparse(q.cuda(), batch, w.cache, mc.Attention(HQ, scale, softcap=cap, window=window), sel.cuda(),
                       count.cuda(), o, w.workspace(mc, T, HQ), lse=lse)
        torch.cuda.synchronize()
        check_rows(w, q, lse.cpu(), [(t, s, j) for t, (s, j) in enumerate(pos)], cap, scale, window, DECODE)


@pytest.mark.parametrize("kind", [BF16, E4M3, E2M1])
@pytest.mark.parametrize("kw", [
    dict(), dict(window=9), dict(window=7), dict(window=2, slopes=True), dict(slopes=True),
    dict(window=33, prefix=[5, 1, 40, 20, 0, 3, 2, 70]), dict(window=20, slopes=True, prefix=[0, 1, 2, 0, 0, 31, 0, 30])])
def test_few_keys_among_many(mc, kind, kw):
    """Rows of one to some hundred keys, random queries: o and lse within the oracle's bounds."""
    w = world(mc, kind, 128)
    if kw.get("slopes"):
        kw = dict(kw, slopes=torch.exp2(-torch.arange(1, HQ + 1).float()))
    for cap in (0.01, 50.0):
        ta.run_attention(mc, w, LENS, HQ, False, cap=cap, what="few", **kw)
        ta.run_attention(mc, w, None, HQ, True, cap=cap, what="few", **kw)
