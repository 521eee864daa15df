"""Edges of the serving calls: every number of pages at which the selection changes how many it holds, attention to
all pages beside attn_decode, and releases of requests whose lengths lie on the borders of pages."""
import random

import pytest

torch = pytest.importorskip("torch")

import test_gpu_attention as ta  # noqa: E402
import test_gpu_sparse as ts  # noqa: E402
from oracle import attention as oa  # noqa: E402
from oracle import cache4 as o4  # noqa: E402
from test_gpu_tables import i32  # noqa: E402

pytestmark = pytest.mark.gpu

mc = ta.mc
BF16, E4M3, E2M1 = ts.BF16, ts.E4M3, ts.E2M1


def select_pages(mc, pages, n_sel, window=0, pool=4, behind=(0, 1000, 7)):
    """Rows at the ends of `pages` pages and before, bounds of a pool of pages (few: many equal scores)."""
    page, D, S = 16, 64, len(behind)
    g = torch.Generator().manual_seed(pages + pool)
    lens = [pages * page - b for b in behind]
    cache = mc.KVCache(pool, page, 1, D)
    table = torch.randint(0, pool, (S, pages), generator=g).to(torch.int32)
    sm = mc.KVSummary(cache)
    sm.bounds.copy_(torch.sort(torch.randint(-127, 128, (pool, 1, 2, D), generator=g), dim=2).values.to(torch.int8))
    sm.scale.copy_(torch.rand((pool, 1), generator=g))
    q = torch.randn((S, 2 * D), generator=g).to(BF16)
    sel = torch.full((S, 1, n_sel), 77, dtype=torch.int32, device="cuda")
    count = torch.full((S, 1), 77, dtype=torch.int32, device="cuda")
    ws = torch.full((mc.attn_select_workspace(S, 1, pages),), 255, dtype=torch.uint8, device="cuda")
    bt = mc.KVBatch(torch.tensor(lens, dtype=torch.int32, device="cuda"), table.cuda())
    print("select", pages, n_sel, window, pool, flush=True)
    mc.attn_select(q.cuda(), bt, cache, sm, mc.Attention(2, 0.125, window=window), sel, count, ws, keep_first=2, keep_last=3)
    b, s = sm.bounds.cpu().long(), sm.scale.cpu()
    for r in range(S):
        at = table[r].long()
        want = o4.select(q[r].float().view(2, D), b[at, 0, 0], b[at, 0, 1], s[at, 0], lens[r] - 1, page, n_sel, 2, 3,
                         window=window)
        assert sel[r, 0].tolist() == want + [-1] * (n_sel - len(want)) and int(count[r, 0]) == len(want), r


@pytest.mark.parametrize("pool", [4, 5000])
@pytest.mark.parametrize("pages", [255, 256, 257, 511, 512, 513, 1023, 1024, 1025, 1500, 2047, 2048, 2049, 2500])
def test_select_counts(mc, pages, pool):
    for n_sel in (5, 64, 254):
        select_pages(mc, pages, n_sel, pool=pool)


@pytest.mark.parametrize("seen", [512, 513, 1024, 1025, 1500, 2048, 2049])
def test_select_behind_a_window(mc, seen):
    """Rows whose window hides the first pages, by whole pages and into one."""
    for window in (16 * seen, 16 * (seen - 1) + 1, 16 * (seen - 1) + 2, 16 * seen - 9):
        select_pages(mc, 3000, 33, window=window, pool=700, behind=(0, 9, 16 * 40))


@pytest.mark.parametrize("kind", [BF16, E4M3, E2M1])
@pytest.mark.parametrize("D,page,kw", [(128, 16, {}), (64, 64, dict(cap=30.0)), (128, 32, dict(window=100)),
                                       (64, 16, dict(cap=80.0, window=700))])
def test_all_pages_are_attn_decode(mc, kind, D, page, kw):
    """All pages listed, in a call of one row a sequence: attn_decode's o and lse within both calls' bounds."""
    lens, g, Hkv = [2000, 777, 1, 0, 64, 33], 4, 2
    w = ts.world(mc, kind, lens, Hkv=Hkv, D=D, page=page, seed=8)
    S, P, Hq, scale = len(lens), w.table.shape[1], 4 * 2, D ** -0.5
    q = w.randn(S, Hq * D).to(BF16)
    sel = torch.arange(P, dtype=torch.int32, device="cuda").repeat(S, Hkv, 1)
    count = torch.tensor([[-(-n // page)] * Hkv for n in lens], dtype=torch.int32, device="cuda")
    bt = ts.batch_of(mc, w, lens)
    at = mc.Attention(Hq, scale, softcap=kw.get("cap", 0.0), window=kw.get("window", 0))
    got = []
    for call in (lambda o, lse: mc.attn_sparse(q.cuda(), bt, w.cache, at, sel, count, o, w.workspace(mc, S, Hq), lse=lse),
                 lambda o, lse: mc.attn_decode(q.cuda(), bt, w.cache, at, o, w.workspace(mc, S, Hq), lse=lse)):
        o, lse = torch.full((S, Hq * D), 7.0, dtype=BF16, device="cuda"), torch.full((S, Hq), 7.0, device="cuda")
        print("all pages", kind, D, page, kw, flush=True)
        call(o, lse)
        got.append((o.cpu().double(), lse.cpu().double()))
    for s, n in enumerate(lens):
        for hq in range(Hq):
            k, v = w.rows("k", s, hq // g, n), w.rows("v", s, hq // g, n)
            _, _, to, tl = oa.attend(q[s:s + 1, hq * D:(hq + 1) * D].double(), k, v, torch.tensor([n - 1]), scale=scale, **kw)
            ta.check(got[0][0][s:s + 1, hq * D:(hq + 1) * D], got[1][0][s:s + 1, hq * D:(hq + 1) * D], 2 * to, "o s=%d" % s)
            ta.check(got[0][1][s:s + 1, hq], got[1][1][s:s + 1, hq], 2 * tl, "lse s=%d" % s)


@pytest.mark.parametrize("S", [8, 64, 1024, 1025, 3000])
@pytest.mark.parametrize("which", ["some", "all", "none"])
@pytest.mark.parametrize("in_place", [False, True])
def test_release_on_borders(mc, S, which, in_place):
    """Ended requests of no token, one, a page, one more or less than pages, their whole row and a negative length;
    any value but 0 of `done` ends one."""
    page, max_pages = 16, 5
    r = random.Random(S)
    past = [(0, 1, page - 1, page, page + 1, 3 * page, max_pages * page, -7)[s % 8] for s in range(S)]
    table = torch.arange(S * max_pages, dtype=torch.int32).view(S, max_pages)
    done = [{"some": r.choice([0, 0, 1, 2, 128, 255]), "all": 1, "none": 0}[which] for _ in range(S)]
    for room in (S * max_pages + 3, 3 * S // 2):                       # the stack takes all, or not all
        free = [-9] * room
        free[:3] = [10 ** 6, 10 ** 6 + 1, 10 ** 6 + 2]
        ref = list(free)
        want_len, height = o4.release(done, past, ref, 3, table, page)
        d_past = i32(past)
        kv_len = d_past if in_place else i32([9] * S)
        pool = mc.KVPool(page, i32(free), i32([3]), None if in_place else i32([0]))
        ws = torch.full((mc.kv_tables_workspace(S),), 255, dtype=torch.uint8, device="cuda")
        d_table = table.cuda()
        print("release", S, which, room, flush=True)
        mc.kv_release(torch.tensor(done, dtype=torch.uint8, device="cuda"), d_past, pool, mc.KVBatch(kv_len, d_table), ws)
        assert kv_len.tolist() == want_len and pool.n_free_out.item() == height
        assert pool.free_list.tolist() == ref and torch.equal(d_table.cpu(), table)
        if which == "none":
            assert want_len == past and height == 3
