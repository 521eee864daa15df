"""Bounds of the pages' keys, selection of pages and attention to them on the GPU, against the
oracle: bounds and selections have to be equal, attention stays within its bounds."""
import pytest

torch = pytest.importorskip("torch")

import test_gpu_attention as ta  # noqa: E402
import test_gpu_cache4 as t4  # noqa: E402
from oracle import cache4 as o4  # noqa: E402

pytestmark = pytest.mark.gpu

mc = ta.mc
BF16, E4M3, E2M1 = torch.bfloat16, torch.float8_e4m3fn, torch.float4_e2m1fn_x2


def world(mc, kind, lens, **kw):
    return t4.World4(mc, lens, **kw) if kind == E2M1 else ta.World(mc, lens, dtype=kind, **kw)


def keys(w, s, h, n):
    """Rows as the bounds see them: of e4m3 the codes' values."""
    k = w.rows("k", s, h, n)
    return k / w.scale["k"][h].double() if getattr(w, "scale", {"k": None})["k"] is not None else k


def bounds_of(w, lens, Hkv):
    """{(page number, head): (lo, hi, scale)} of all pages of the sequences."""
    out = {}
    for s, n in enumerate(lens):
        for h in range(Hkv):
            k = keys(w, s, h, n).float()
            for p in range(-(-n // w.page)):
                out[int(w.table[s, p]), h] = o4.bounds(k[p * w.page:(p + 1) * w.page])
    return out


def batch_of(mc, w, lens, new=None, T=None):
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if new is None:
        return mc.KVBatch(kv_len, w.table.cuda())
    return mc.KVBatch(kv_len, w.table.cuda(), q_start=ta.starts(new), T=T or sum(new))


def summarize_all(mc, w, lens):
    sm = mc.KVSummary(w.cache)
    sm.bounds.fill_(99)
    sm.scale.fill_(99.0)
    new = [n for n in lens]
    mc.kv_summarize(batch_of(mc, w, lens, new), w.cache, sm)
    return sm


@pytest.mark.parametrize("kind", [BF16, E4M3, E2M1])
@pytest.mark.parametrize("D,Hkv,page", [(128, 2, 16), (64, 3, 64), (128, 1, 256), (64, 2, 32)])
def test_summary(mc, kind, D, Hkv, page):
    lens = [1, 300, 64, 17, 0, 513]
    w = world(mc, kind, lens, Hkv=Hkv, D=D, page=page, seed=D)
    sm = summarize_all(mc, w, lens)
    want = bounds_of(w, lens, Hkv)
    got_b, got_s = sm.bounds.cpu().long(), sm.scale.cpu()
    for (p, h), (lo, hi, s) in want.items():
        assert float(got_s[p, h]) == float(s) and torch.equal(got_b[p, h, 0], lo) and torch.equal(got_b[p, h, 1], hi), (p, h)
    others = torch.ones(got_s.shape, dtype=torch.bool)
    for p, h in want:
        others[p, h] = False
    assert bool((got_s[others] == 99.0).all()) and bool((got_b[others] == 99).all())
    # only the pages of the new tokens are renewed
    new = [1, 70, 0, 2, 0, 1]
    for touched, bt in (([(s, p) for s, n in enumerate(new) for p in range((lens[s] - n) // page, -(-lens[s] // page)) if n],
                         batch_of(mc, w, lens, new, T=sum(new) + 5)),
                        ([(s, (n - 1) // page) for s, n in enumerate(lens) if n], batch_of(mc, w, lens))):
        sm.bounds.fill_(5)
        sm.scale.fill_(5.0)
        mc.kv_summarize(bt, w.cache, sm)
        pages = {int(w.table[s, p]) for s, p in touched}
        for p in range(sm.scale.shape[0]):
            for h in range(Hkv):
                if p in pages:
                    assert float(sm.scale[p, h]) == float(want[p, h][2])
                    assert torch.equal(sm.bounds[p, h].cpu().long(), torch.stack(want[p, h][:2]))
                else:
                    assert float(sm.scale[p, h]) == 5.0 and bool((sm.bounds[p, h] == 5).all())


def test_summary_leaves_out_what_is_no_number(mc):
    w = ta.World(mc, [40], Hkv=1, D=64, page=16, odd=[(0, 3, 0, 5, "k", float("nan")), (0, 4, 0, 6, "k", float("inf"))]
                 + [(0, j, 0, i, "k", float("-inf")) for j in range(16, 32) for i in range(64)])
    sm = summarize_all(mc, w, [40])
    for p, want in ((p, bounds_of(w, [40], 1)[int(w.table[0, p]), 0]) for p in range(3)):
        at = int(w.table[0, p])
        assert float(sm.scale[at, 0]) == float(want[2]) and torch.equal(sm.bounds[at, 0].cpu().long(), torch.stack(want[:2]))
    assert float(sm.scale[int(w.table[0, 1]), 0]) == 0.0


def tables_of(w, want, s, h, n):
    got = [want[int(w.table[s, p]), h] for p in range(-(-n // w.page))]
    return torch.stack([x[0] for x in got]), torch.stack([x[1] for x in got]), torch.stack([x[2] for x in got])


def check_selection(w, want, q, lens, new, Hq, Hkv, n_sel, first, last, sel, count, window=0, negative=False):
    g, t = Hq // Hkv, 0
    for s, n in enumerate(new):
        for r in range(n):
            pos = lens[s] - n + r
            for h in range(Hkv):
                lo, hi, sc = tables_of(w, want, s, h, lens[s])
                qr = q[t, h * g * w.D:(h + 1) * g * w.D].float().view(g, w.D)
                exp = o4.select(qr, lo, hi, sc, pos, w.page, n_sel, first, last, window, negative)
                got = sel[t, h].tolist()
                assert int(count[t, h]) == len(exp) and got == exp + [-1] * (n_sel - len(exp)), (s, r, h)
            t += 1


@pytest.mark.parametrize("kind,D,Hq,Hkv,page,n_sel,first,last,window", [
    (BF16, 128, 8, 2, 16, 8, 1, 2, 0), (E4M3, 64, 6, 2, 32, 3, 0, 1, 0), (E2M1, 128, 5, 1, 16, 5, 1, 1, 200),
    (BF16, 64, 20, 1, 16, 6, 2, 3, 0), (E2M1, 64, 3, 3, 64, 1, 0, 1, 0), (BF16, 128, 32, 1, 16, 9, 0, 9, 0),
    (BF16, 128, 2, 2, 16, 300, 1, 1, 0), (E4M3, 128, 16, 1, 16, 7, 6, 1, 0)])
def test_select_and_attend(mc, kind, D, Hq, Hkv, page, n_sel, first, last, window):
    lens, new = [700, 33, 0, 150, 290], [40, 3, 0, 1, 19]
    w = world(mc, kind, lens, Hkv=Hkv, D=D, page=page, seed=n_sel)
    sm = summarize_all(mc, w, lens)
    want = bounds_of(w, lens, Hkv)
    T, pad = sum(new), 2
    q = w.randn(T + pad, Hq * D + 8).to(BF16)
    q[2, 5], q[3, 70], q[4] = float("nan"), float("inf"), 0
    qd = q.cuda()[:, :Hq * D]
    bt = batch_of(mc, w, lens, new, T=T + pad)
    for scale in (D ** -0.5, -D ** -0.5):
        at = mc.Attention(Hq, scale, window=window, softcap=30.0)
        sel = torch.full((T + pad, Hkv, n_sel), 77, dtype=torch.int32, device="cuda")
        count = torch.full((T + pad, Hkv), 77, dtype=torch.int32, device="cuda")
        ws = torch.full((max(mc.attn_select_workspace(T + pad, Hkv, w.table.shape[1]), mc.attn_workspace(T + pad, Hq, Hkv, D)),),
                        255, dtype=torch.uint8, device="cuda")
        print("select", kind, D, Hq, Hkv, flush=True)
        mc.attn_select(qd, bt, w.cache, sm, at, sel, count, ws, keep_first=first, keep_last=last)
        torch.cuda.synchronize()
        assert bool((sel[T:] == 77).all()) and bool((count[T:] == 77).all())
        check_selection(w, want, q[:, :Hq * D], lens, new, Hq, Hkv, n_sel, first, last, sel.cpu(), count.cpu(), window,
                        scale < 0)
    q[2, 5], q[3, 70] = 1.0, 1.0
    qd = q.cuda()[:, :Hq * D]
    check_sparse(mc, w, q[:, :Hq * D], qd, bt, lens, new, Hq, Hkv, sel, count, pad, scale=-D ** -0.5, window=window, cap=30.0)


def check_sparse(mc, w, q, qd, bt, lens, new, Hq, Hkv, sel, count, pad=0, scale=0.1, window=0, cap=0.0, slopes=None):
    T, D, g, page = sum(new), w.D, Hq // Hkv, w.page
    o = torch.full((T + pad, Hq * D + 8), 7.0, dtype=BF16, device="cuda")
    lse = torch.full((T + pad, Hq), 7.0, device="cuda")
    at = mc.Attention(Hq, scale, softcap=cap, window=window, slopes=None if slopes is None else slopes.cuda())
    print("sparse", T, Hq, Hkv, tuple(sel.shape), flush=True)
    mc.attn_sparse(qd, bt, w.cache, at, sel, count, o[:, :Hq * D], w.workspace(mc, T + pad, Hq), lse=lse)
    torch.cuda.synchronize()
    assert bool((o[:, Hq * D:] == 7.0).all()) and bool((o[T:] == 7.0).all()) and bool((lse[T:] == 7.0).all())
    oc, lc, sc, cc = o.cpu(), lse.cpu(), sel.cpu(), count.cpu()
    rows = {(s, h): (w.rows("k", s, h, n), w.rows("v", s, h, n)) for s, n in enumerate(lens) for h in range(Hkv)}
    t = 0
    for s, n in enumerate(new):
        for r in range(n):
            pos = lens[s] - n + r
            for h in range(Hkv):
                k, v = rows[s, h]
                times = torch.zeros(lens[s], dtype=torch.int64)
                for p in sc[t, h, :max(0, min(int(cc[t, h]), sel.shape[2]))].tolist():
                    if 0 <= p < w.table.shape[1]:
                        times[p * page:(p + 1) * page] += 1
                for hq in range(h * g, (h + 1) * g):
                    ro, rl, to, tl = o4.attend_some(q[t:t + 1, hq * D:(hq + 1) * D].double(), k, v, pos, times, scale=scale,
                                                    cap=cap, window=window,
                                                    slope=0.0 if slopes is None else float(slopes[hq]))
                    ta.check(oc[t:t + 1, hq * D:(hq + 1) * D], ro, to, "o s=%d r=%d hq=%d" % (s, r, hq))
                    ta.check(lc[t:t + 1, hq], rl, tl, "lse s=%d r=%d hq=%d" % (s, r, hq))
            t += 1


@pytest.mark.parametrize("kind,D,Hkv,page,g", [(BF16, 128, 2, 16, 4), (E4M3, 64, 2, 16, 1), (E2M1, 128, 1, 16, 3),
                                               (E2M1, 64, 2, 64, 20), (BF16, 64, 1, 256, 2), (E4M3, 128, 1, 128, 17)])
def test_sparse_lists(mc, kind, D, Hkv, page, g):
    """Lists in any order, with gaps, twice the same, out of the table, behind the row, empty and cut by count;
    one row a sequence and ragged ones."""
    lens = [600, 1, 40, 0, 333]
    w = world(mc, kind, lens, Hkv=Hkv, D=D, page=page, seed=page + g, gap=1)
    Hq, n_sel = Hkv * g, 6
    P = w.table.shape[1]
    gen = torch.Generator().manual_seed(1)
    slopes = torch.exp2(-torch.arange(1, Hq + 1).float() / 4)
    for new in (None, [9, 1, 3, 0, 2]):
        rows = len(lens) if new is None else sum(new)
        sel = torch.stack([torch.randperm(max(P, n_sel), generator=gen)[:n_sel] for _ in range(rows * Hkv)])
        sel = sel.view(rows, Hkv, n_sel).to(torch.int32)
        sel[0, 0] = torch.tensor([0, 0, -1, P, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
        count = torch.randint(1, n_sel + 1, (rows, Hkv), generator=gen).to(torch.int32)
        count[0, 0] = n_sel + 5
        count[1 % rows, 0] = 0
        count[2 % rows, 0] = -4
        q = w.randn(rows, Hq * D).to(BF16)
        bt = batch_of(mc, w, lens, new)
        args = dict(scale=D ** -0.5)
        for kw in (dict(), dict(window=50), dict(cap=0.7, slopes=slopes), dict(slopes=slopes, window=300)):
            check_sparse(mc, w, q, q.cuda(), bt, lens, new or [1] * len(lens), Hq, Hkv, sel.cuda(), count.cuda(), **args,
                         **kw)


@pytest.mark.parametrize("kind", [BF16, E4M3, E2M1])
def test_sparse_of_all_pages_is_decode(mc, kind):
    """All pages listed: what attn_decode gives, within the bound of both; and split over the list."""
    lens = [2000, 777]
    w = world(mc, kind, lens, Hkv=1, D=128, page=16, seed=8)
    P = w.table.shape[1]
    sel = torch.arange(P, dtype=torch.int32).repeat(2, 1, 1)
    count = torch.tensor([[125], [49]], dtype=torch.int32)
    q = w.randn(2, 4 * 128).to(BF16)
    check_sparse(mc, w, q, q.cuda(), batch_of(mc, w, lens), lens, [1, 1], 4, 1, sel.cuda(), count.cuda(), scale=0.09)


@pytest.mark.parametrize("pages,n_sel", [(9000, 33), (700, 256), (8192, 4096)])
def test_select_of_many_pages(mc, pages, n_sel):
    """More pages than are held at once, equal scores by the lower page; bounds are given."""
    page, D = 16, 64
    g = torch.Generator().manual_seed(pages)
    lens = [pages * page, pages * page - 1000]
    cache = mc.KVCache(4, page, 1, D, k=torch.zeros((4, page * D), dtype=BF16, device="cuda"),
                       v=torch.zeros((4, page * D), dtype=BF16, device="cuda"))
    table = torch.randint(0, 4, (2, pages), generator=g).to(torch.int32)         # (a page many times: many equal scores)
    sm = mc.KVSummary(cache)
    lo = torch.randint(-127, 128, (4, 1, 2, D), generator=g)
    sm.bounds.copy_(torch.sort(lo, dim=2).values.to(torch.int8))
    sm.scale.copy_(torch.rand((4, 1), generator=g))
    q = torch.randn((2, 2 * D), generator=g).to(BF16)
    sel = torch.empty((2, 1, n_sel), dtype=torch.int32, device="cuda")
    count = torch.empty((2, 1), dtype=torch.int32, device="cuda")
    ws = torch.empty(mc.attn_select_workspace(2, 1, pages), dtype=torch.uint8, device="cuda")
    bt = mc.KVBatch(torch.tensor(lens, dtype=torch.int32, device="cuda"), table.cuda())
    mc.attn_select(q.cuda(), bt, cache, sm, mc.Attention(2, 0.125), sel, count, ws, keep_first=2, keep_last=3)
    b, s = sm.bounds.cpu().long(), sm.scale.cpu()
    for r in range(2):
        at = table[r].long()
        want = o4.select(q[r].float().view(2, D), b[at, 0, 0], b[at, 0, 1], s[at, 0], lens[r] - 1, page, n_sel, 2, 3)
        assert sel[r, 0].tolist() == want and int(count[r, 0]) == n_sel


def test_select_in_parts(mc):
    """More scores than the workspace's 256 MB: the rows go in parts."""
    page, D, pages, T = 16, 64, 65536, 1100
    cache = mc.KVCache(2, page, 1, D)
    g = torch.Generator().manual_seed(0)
    table = torch.randint(0, 2, (1, pages), generator=g).to(torch.int32)
    sm = mc.KVSummary(cache)
    sm.bounds.copy_(torch.sort(torch.randint(-127, 128, (2, 1, 2, D), generator=g), dim=2).values.to(torch.int8))
    sm.scale.fill_(0.5)
    q = torch.randn((T, D), generator=g).to(BF16)
    n = pages * page
    bt = mc.KVBatch(torch.tensor([n], dtype=torch.int32, device="cuda"), table.cuda(), q_start=ta.starts([T]), T=T)
    sel = torch.full((T, 1, 5), -9, dtype=torch.int32, device="cuda")
    count = torch.empty((T, 1), dtype=torch.int32, device="cuda")
    need = mc.attn_select_workspace(T, 1, pages)
    assert need == 256 << 20
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    mc.attn_select(q.cuda(), bt, cache, sm, mc.Attention(1, 0.125), sel, count, ws)
    b, s, at = sm.bounds.cpu().long(), sm.scale.cpu(), table[0].long()
    for t in (0, 1, 511, 1023, 1024, 1025, T - 1):
        want = o4.select(q[t:t + 1].float(), b[at, 0, 0], b[at, 0, 1], s[at, 0], n - T + t, page, 5, 1, 1)
        assert sel[t, 0].tolist() == want, t
    assert bool((count == 5).all())
