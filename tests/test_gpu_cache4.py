"""A cache held in 4 bits on the GPU, against the 64-bit oracle: append, read, decode, prefill and
importance.  Every place of the cache that no sequence holds is NaN; codes and scales have to be
the oracle's, attention stays within its bounds."""
import pytest

torch = pytest.importorskip("torch")

import test_gpu_attention as ta  # noqa: E402
from oracle import attention as oa  # noqa: E402
from oracle import cache4 as o4  # noqa: E402

pytestmark = pytest.mark.gpu

mc = ta.mc
BF16, E2M1 = torch.bfloat16, torch.float4_e2m1fn_x2


class World4:
    """As test_gpu_attention's World, its pages e2m1."""

    def __init__(self, mc, lens, Hkv=2, D=128, page=16, seed=0, gap=0, extra_pages=2, loud=()):
        g = torch.Generator().manual_seed(seed)
        self.gen, self.lens, self.Hkv, self.D, self.page, self.dtype = g, lens, Hkv, D, page, E2M1
        used = [-(-n // page) for n in lens]
        self.n_pages = sum(used) + extra_pages
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), max(1, max(used)) + gap), -7, dtype=torch.int32)
        at = 0
        for s, u in enumerate(used):
            self.table[s, :u] = order[at:at + u]
            at += u
        per = o4.page_bytes(page, Hkv, D)
        self.flat = {w: torch.full((self.n_pages, per), 255, dtype=torch.uint8) for w in "kv"}
        for w in "kv":
            for s, n in enumerate(lens):
                for h in range(Hkv):
                    x = torch.randn((n, D), generator=g) * torch.exp(0.5 * torch.randn((n, 1), generator=g))
                    for (ls, lj, lw, val) in loud:
                        if (ls, lw) == (s, w):
                            x[lj] = val
                    codes, scale = (o4.quantize_keys if w == "k" else o4.quantize_values)(x.to(BF16))
                    o4.write(w, self.flat[w], self.table[s], torch.arange(n), h, codes, scale, page, Hkv, D)
        self.cache = mc.KVCache(self.n_pages, page, Hkv, D, dtype=E2M1, k=self.flat["k"].cuda(),
                                v=self.flat["v"].cuda())

    def rows(self, w, s, h, n=None):
        return o4.read(w, self.flat[w], self.table[s], self.lens[s] if n is None else n, h, self.page, self.Hkv, self.D)

    def randn(self, *shape):
        return torch.randn(shape, generator=self.gen)

    def workspace(self, mc, T, Hq):
        return torch.full((mc.attn_workspace(T, Hq, self.Hkv, self.D),), 255, dtype=torch.uint8, device="cuda")


def quiet_zeros(flat):
    """Bytes with codes of -0 as 0."""
    lo, hi = flat & 15, flat >> 4
    lo, hi = (torch.where(x == 8, torch.zeros_like(x), x) for x in (lo, hi))
    return lo | (hi << 4)


# ------------------------------------------------------------------ append --

@pytest.mark.parametrize("D,Hq,Hkv,page,norm,rot,pairs", [
    (128, 4, 2, 16, "none", 128, False),
    (64, 6, 2, 32, "head", 64, True),
    (128, 3, 3, 64, "row", 128, False),
    (128, 8, 2, 16, "head", 64, False),
    (64, 16, 16, 256, "row", 32, True),
    (64, 1, 1, 128, "none", 0, False),
    (128, 12, 4, 16, "row", 16, True),
    (64, 0, 2, 16, "head", 48, False),       # keys and values alone
    (128, 40, 1, 32, "none", 128, True),
    (128, 40, 8, 16, "row", 128, False),     # rows of more than a wave holds
    (128, 96, 32, 32, "row", 64, True),
    (64, 5, 256, 16, "head", 64, False),
])
def test_append(mc, D, Hq, Hkv, page, norm, rot, pairs):
    new = [1, 0, 37, 16, 5, 32, 1, 8, 2]
    lens = [1, 9, 40, 32, 100, 64, 50, 15, 33]
    w = World4(mc, lens, Hkv=Hkv, D=D, page=page, seed=D + Hq)
    T = sum(new)
    qkv = (w.randn(T + 2, (Hq + 2 * Hkv) * D) * torch.exp(w.randn(T + 2, 1))).to(BF16)
    edge = qkv[:, Hq * D:]
    edge[3] = 0                               # a token of zeros, of one large number, NaN, infinite, tiny, huge
    edge[5, 7::64] = 1000.0
    edge[9, 3], edge[10, Hkv * D + 70 % D] = float("nan"), float("inf")
    edge[20] *= 2.0 ** -110
    edge[21, Hkv * D:] = 2.0 ** 127.9 if norm == "none" and not rot else 3.0
    rope = torch.stack((torch.cos(w.randn(300, max(rot // 2, 1))), torch.sin(w.randn(300, max(rot // 2, 1)))), -1)
    width = {"none": 0, "head": D, "row": -1}[norm]
    wq, wk = ((1 + 0.2 * w.randn(h * D if width < 0 else D)).to(BF16) if width else None for h in (max(Hq, 1), Hkv))
    prep = mc.QKPrep(rope=rope.cuda() if rot else None, rope_pairs=pairs, q_norm=None if wq is None else wq.cuda(),
                     k_norm=None if wk is None else wk.cuda(), norm_row=norm == "row", eps=1e-6)
    batch = mc.KVBatch(torch.tensor(lens, dtype=torch.int32, device="cuda"), w.table.cuda(), q_start=ta.starts(new),
                       T=T + 2)
    d = qkv.cuda()
    out = torch.full((T + 2, Hq * D + 8), 7.0, dtype=BF16, device="cuda")
    print("append", D, Hq, Hkv, page, norm, flush=True)
    mc.kv_append(d[:, :Hq * D] if Hq else None, d[:, Hq * D:(Hq + Hkv) * D], d[:, (Hq + Hkv) * D:], prep, batch,
                 w.cache, out[:, :Hq * D] if Hq else None)
    k_read, v_read = (torch.full((T + 2, Hkv * D + 16), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    mc.kv_read(batch, w.cache, k_read[:, :Hkv * D], v_read[:, :Hkv * D])
    torch.cuda.synchronize()
    assert bool((out[T:] == 7.0).all()) and bool((out[:, Hq * D:] == 7.0).all())
    for x in (k_read, v_read):
        assert bool((x[T:] == 7.0).all()) and bool((x[:, Hkv * D:] == 7.0).all())
    want = {x: w.flat[x].clone() for x in "kv"}
    t0, eps = 0, float(torch.tensor(1e-6))
    for s, n in enumerate(new):
        if n == 0:
            continue
        pos = lens[s] - n + torch.arange(n)
        x = qkv[t0:t0 + n].double()
        args = (norm, eps, rot, pairs, rope[pos].double())
        if Hq:
            yq, eq = oa.prepare(x[:, :Hq * D], Hq, D, None if wq is None else wq.double(), *args)
            ta.check(out[t0:t0 + n, :Hq * D].cpu().view(n, Hq, D), yq, oa.BF * (yq.abs() + eq) + eq, "q_out s=%d" % s)
        yk, _ = oa.prepare(x[:, Hq * D:(Hq + Hkv) * D], Hkv, D, None if wk is None else wk.double(), *args)
        yv = x[:, (Hq + Hkv) * D:].view(n, Hkv, D)
        for which, y, got in (("k", yk, k_read), ("v", yv, v_read)):
            codes, scale = (o4.quantize_keys if which == "k" else o4.quantize_values)(y)
            for h in range(Hkv):
                o4.write(which, want[which], w.table[s], pos, h, codes[:, h], scale[:, h], page, Hkv, D)
                val = o4.values(which, codes[:, h], scale[:, h])
                g = got[t0:t0 + n, h * D:(h + 1) * D].double().cpu()
                assert torch.equal(torch.isnan(g), torch.isnan(val)) and torch.equal(torch.nan_to_num(g), torch.nan_to_num(val)), \
                    "%s read s=%d h=%d" % (which, s, h)
        t0 += n
    for x in "kv":     # all bytes: the new tokens', and everything else as it was
        got, exp = quiet_zeros(getattr(w.cache, x).cpu()), quiet_zeros(want[x])
        assert torch.equal(got, exp), (x, [(*i, int(got[tuple(i)]), int(exp[tuple(i)])) for i in (got != exp).nonzero()[:9].tolist()])


@pytest.mark.parametrize("D,page", [(64, 16), (128, 32)])
def test_append_one_by_one(mc, D, page):
    """Tokens appended one a call leave what all at once leave."""
    Hkv, n = 2, 37
    g = torch.Generator().manual_seed(5)
    k, v = (torch.randn((n, Hkv * D), generator=g).to(BF16).cuda() for _ in range(2))
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device="cuda")
    caches = [mc.KVCache(3, page, Hkv, D, dtype=E2M1) for _ in range(2)]
    batch = mc.KVBatch(torch.tensor([n], dtype=torch.int32, device="cuda"), table, q_start=ta.starts([n]), T=n)
    mc.kv_append(None, k, v, None, batch, caches[0], None)
    kv_len = torch.zeros(1, dtype=torch.int32, device="cuda")
    one = mc.KVBatch(kv_len, table, q_start=ta.starts([1]), T=1)
    for i in range(n):
        kv_len += 1
        mc.kv_append(None, k[i:i + 1], v[i:i + 1], None, one, caches[1], None)
    for x in "kv":
        assert torch.equal(getattr(caches[0], x), getattr(caches[1], x)), x


def test_append_skips(mc):
    """Tokens without a page, behind the table or past the rotation table leave everything as it was."""
    D, Hkv, page = 64, 1, 16
    w = World4(mc, [16], Hkv=Hkv, D=D, page=page, extra_pages=3)
    table = torch.tensor([[0, 99], [-1, 1], [2, 2]], dtype=torch.int32, device="cuda")
    kv_len = torch.tensor([20, 3, 50], dtype=torch.int32, device="cuda")
    new = [4, 3, 18]
    rope = torch.ones((31, 32, 2), device="cuda")
    batch = mc.KVBatch(kv_len, table, q_start=ta.starts(new), T=25)
    x = torch.ones((25, D), dtype=BF16, device="cuda")
    before = {a: getattr(w.cache, a).clone() for a in "kv"}
    mc.kv_append(None, x, x, mc.QKPrep(rope=rope), batch, w.cache, None)
    # (kv_len 50 is cut to the table's 32: positions 32 to 49 are past it)
    for a in "kv":
        assert torch.equal(getattr(w.cache, a), before[a])
    out = torch.full((25, D), 7.0, dtype=BF16, device="cuda")
    mc.kv_read(batch, w.cache, out, None)
    assert bool((out == 7.0).all())


@pytest.mark.parametrize("dtype", [BF16, torch.float8_e4m3fn])
def test_read_of_the_other_kinds(mc, dtype):
    """bf16 as it is, e4m3 times its scale."""
    lens, new = [40, 7, 100], [33, 0, 50]
    w = ta.World(mc, lens, Hkv=3, D=64, page=32, dtype=dtype, seed=3)
    T = sum(new)
    batch = mc.KVBatch(torch.tensor(lens, dtype=torch.int32, device="cuda"), w.table.cuda(), q_start=ta.starts(new), T=T)
    k, v = (torch.empty((T, 3 * 64), dtype=BF16, device="cuda") for _ in range(2))
    mc.kv_read(batch, w.cache, k, v)
    t0 = 0
    for s, n in enumerate(new):
        for which, got in (("k", k), ("v", v)):
            for h in range(3):
                # (the product of a code and an fp32 scale is exact in 64 bits; it is rounded to fp32, then to bf16)
                want = w.rows(which, s, h)[lens[s] - n:].float().to(BF16)
                assert torch.equal(got[t0:t0 + n, h * 64:(h + 1) * 64].cpu(), want), (which, s, h)
        t0 += n


# --------------------------------------------------------------- attention --

@pytest.mark.parametrize("D,Hq,Hkv,page", [(128, 8, 2, 16), (64, 6, 2, 32), (128, 5, 5, 64), (64, 40, 1, 16),
                                           (128, 3, 1, 256), (64, 32, 32, 16)])
def test_decode(mc, D, Hq, Hkv, page):
    lens = [1, 2, 15, 16, 17, 64, 65, 300, 0, 511]
    w = World4(mc, lens, Hkv=Hkv, D=D, page=page, seed=Hq)
    ta.run_attention(mc, w, [1] * len(lens), Hq, True, what="decode", wide=8)


@pytest.mark.parametrize("kw", [
    dict(window=40), dict(window=1), dict(cap=20.0), dict(cap=0.5), dict(cap=200.0), dict(slopes=True), dict(prefix=[5, 0, 400, 16]),
    dict(window=33, prefix=[70, 3, 0, 20], cap=30.0, slopes=True)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("decode", [True, False])
def test_masks(mc, D, kw, decode):
    lens, new = [333, 70, 260, 64], [100, 1, 0, 64]
    w = World4(mc, lens, Hkv=2, D=D, page=16, seed=7)
    kw = dict(kw)
    if kw.get("slopes"):
        kw["slopes"] = torch.exp2(-torch.arange(1, 5).float())
    ta.run_attention(mc, w, new, 4, decode, what=str(kw), **kw)


@pytest.mark.parametrize("S,n", [(1, 5000), (3, 1500), (40, 90)])
def test_decode_split(mc, S, n):
    lens = [n - 37 * i for i in range(S)] if S < 10 else [n - i for i in range(S)]
    w = World4(mc, lens, Hkv=2, D=128, page=64, seed=S)
    ta.run_attention(mc, w, [1] * S, 8, True, max_len=n, what="split")


@pytest.mark.parametrize("D,Hq,Hkv,page", [(128, 8, 2, 16), (64, 4, 2, 32), (64, 6, 1, 64), (128, 2, 2, 256)])
def test_prefill(mc, D, Hq, Hkv, page):
    lens, new = [1, 130, 77, 64, 200, 9, 0], [1, 130, 40, 64, 3, 9, 0]
    w = World4(mc, lens, Hkv=Hkv, D=D, page=page, seed=D)
    ta.run_attention(mc, w, new, Hq, False, what="prefill", wide=16)


@pytest.mark.parametrize("D", [64, 128])
def test_prefill_long(mc, D):
    """Splits, two teams of waves, offsets of more than 64 tiles."""
    w = World4(mc, [4700], Hkv=1, D=D, page=128, seed=1)
    ta.run_attention(mc, w, [40], 2, False, what="long chunk")
    w = World4(mc, [700], Hkv=2, D=D, page=32, seed=2)
    ta.run_attention(mc, w, [700], 2, False, what="prompt")


@pytest.mark.parametrize("decode", [True, False])
@pytest.mark.parametrize("D", [64, 128])
def test_nan_reaches_only_those_that_see_it(mc, D, decode):
    """A token whose values or keys are NaN: rows that see it, and no others, are NaN."""
    lens, new = [100, 90], [100, 90]
    w = World4(mc, lens, Hkv=1, D=D, page=16, seed=4, loud=[(0, 60, "v", float("nan")), (1, 50, "k", float("inf"))])
    q = w.randn(192, 2 * D).to(BF16)
    o = torch.empty((192, 2 * D), dtype=BF16, device="cuda")
    lse = torch.empty((192, 2), device="cuda")
    ws = w.workspace(mc, 192, 2)
    table = w.table.cuda()
    for window in (0, 20):
        at = mc.Attention(2, D ** -0.5, window=window)
        if decode:
            for a in (59, 60, 61, 85, 90):
                kv_len = torch.tensor([a, a], dtype=torch.int32, device="cuda")
                mc.attn_decode(q[:2].cuda(), mc.KVBatch(kv_len, table), w.cache, at, o[:2], ws, lse=lse[:2])
                sees = (a > 60 and (not window or a - 1 - 60 < window), a > 50 and (not window or a - 1 - 50 < window))
                assert (bool(torch.isnan(o[0]).all()), bool(torch.isnan(o[1]).all())) == sees, a
                assert (bool(torch.isnan(o[0]).any()), bool(torch.isnan(o[1]).any())) == sees, a
            continue
        batch = mc.KVBatch(torch.tensor(lens, dtype=torch.int32, device="cuda"), table, q_start=ta.starts(new), T=190)
        mc.attn_prefill(q[:190].cuda(), batch, w.cache, at, o[:190], ws, lse=lse[:190])
        i = torch.arange(100)
        want = torch.cat(((i >= 60) & ((i < 60 + window) | (window == 0)),
                          ((i >= 50) & ((i < 50 + window) | (window == 0)))[:90]))
        got = torch.isnan(o[:190]).cpu()
        assert torch.equal(got.all(1), want) and torch.equal(got.any(1), want)


@pytest.mark.parametrize("D,Hq,Hkv,kw", [(128, 4, 2, {}), (64, 2, 1, dict(window=50)), (128, 3, 3, dict(softcap=20.0))])
def test_importance(mc, D, Hq, Hkv, kw):
    L, d = 333, 128
    w = World4(mc, [L], Hkv=Hkv, D=D, page=32, seed=9)
    q = w.randn(L, Hq * D).to(BF16)
    x = w.randn(L, d).to(BF16)
    batch = mc.KVBatch(torch.tensor([L], dtype=torch.int32, device="cuda"), w.table.cuda(), q_start=ta.starts([L]), T=L)
    at = mc.Attention(Hq, D ** -0.5, **kw)
    o = torch.empty((L, Hq * D), dtype=BF16, device="cuda")
    lse = torch.empty((L, Hq), device="cuda")
    ws = torch.empty(max(mc.attn_workspace(L, Hq, Hkv, D), mc.attn_importance_workspace(Hq, L)), dtype=torch.uint8,
                     device="cuda")
    mc.attn_prefill(q.cuda(), batch, w.cache, at, o, ws, lse=lse)
    imp, mask = torch.empty(L, device="cuda"), torch.empty(L, dtype=torch.uint8, device="cuda")
    mc.attn_importance(q.cuda(), lse, batch, w.cache, at, x.cuda(), 0.1, mask, ws, importance=imp)
    keys = [w.rows("k", 0, h) for h in range(Hkv)]
    want, rel = oa.importance(q.double(), lse.double().cpu(), keys, x.double(), L, Hq // Hkv, Hkv, D, scale=D ** -0.5,
                              cap=kw.get("softcap", 0.0), window=kw.get("window", 0))
    ta.check(imp, want, rel * want.abs(), "importance")
    n = int(0.1 * L + 0.5)
    assert int(mask.sum()) == n
    order = torch.sort(imp.cpu(), descending=True, stable=True).indices[:n]
    assert bool(mask.cpu()[order].all())


def test_shared_allocation(mc):
    """Layers that share an allocation: pages with other layers' bytes between them."""
    D, Hkv, page, lens = 128, 2, 16, [100, 40]
    w = World4(mc, lens, Hkv=Hkv, D=D, page=page, seed=11)
    per = o4.page_bytes(page, Hkv, D)
    both = torch.full((w.n_pages, 2, 2, per), 255, dtype=torch.uint8, device="cuda")
    both[:, 1, 0], both[:, 1, 1] = w.flat["k"].cuda(), w.flat["v"].cuda()
    plain = w.cache
    w.cache = mc.KVCache(w.n_pages, page, Hkv, D, dtype=E2M1, k=both[:, 1, 0], v=both[:, 1, 1])
    for decode in (True, False):
        ta.run_attention(mc, w, [60, 40], 4, decode, what="shared")
    batch = mc.KVBatch(torch.tensor(lens, dtype=torch.int32, device="cuda"), w.table.cuda(), q_start=ta.starts([60, 7]),
                       T=67)
    k = w.randn(67, Hkv * D).to(BF16).cuda()
    for cache in (w.cache, plain):
        mc.kv_append(None, k, k, None, batch, cache, None)
    assert torch.equal(both[:, 1, 0], plain.k) and torch.equal(both[:, 1, 1], plain.v)
    assert bool((both[:, 0] == 255).all())


def test_far_pages(mc):
    """Pages behind the first 4 GB: what near pages give, bit for bit."""
    D, Hkv, page, n, Hq = 128, 8, 256, 700, 16
    per = o4.page_bytes(page, Hkv, D)
    n_pages = 2 ** 32 // per + 10
    cache = mc.KVCache(n_pages, page, Hkv, D, dtype=E2M1)
    sm = mc.KVSummary(cache)
    g = torch.Generator().manual_seed(2)
    k, v, q = (torch.randn((n, h * D), generator=g).to(BF16).cuda() for h in (Hkv, Hkv, Hq))
    at = mc.Attention(Hq, D ** -0.5)
    ws = torch.empty(max(mc.attn_workspace(n, Hq, Hkv, D), mc.attn_select_workspace(n, Hkv, 3)), dtype=torch.uint8,
                     device="cuda")
    outs = []
    for table in ([2, 0, 1], [n_pages - 1, n_pages - 3, n_pages - 2]):
        table = torch.tensor([table], dtype=torch.int32, device="cuda")
        kv_len = torch.tensor([n], dtype=torch.int32, device="cuda")
        batch = mc.KVBatch(kv_len, table, q_start=ta.starts([n]), T=n)
        mc.kv_append(None, k, v, None, batch, cache, None)
        mc.kv_summarize(batch, cache, sm)
        back = [torch.empty((n, Hkv * D), dtype=BF16, device="cuda") for _ in range(2)]
        mc.kv_read(batch, cache, *back)
        o, o1, o2 = (torch.empty((n, Hq * D), dtype=BF16, device="cuda") for _ in range(3))
        mc.attn_prefill(q, batch, cache, at, o, ws)
        mc.attn_decode(q[:1], mc.KVBatch(kv_len, table), cache, at, o1[:1], ws)
        sel = torch.empty((n, Hkv, 2), dtype=torch.int32, device="cuda")
        count = torch.empty((n, Hkv), dtype=torch.int32, device="cuda")
        mc.attn_select(q, batch, cache, sm, at, sel, count, ws)
        mc.attn_sparse(q, batch, cache, at, sel, count, o2, ws)
        pages = table[0].long()
        outs.append([*back, o, o1[:1], o2, sel, count, cache.k[pages], cache.v[pages], sm.bounds[pages], sm.scale[pages]])
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert bool((cache.k[3:n_pages - 3] == 0).all()) and float(outs[0][2].float().abs().max()) > 0


@pytest.mark.parametrize("D", [64, 128])
def test_rows_before_the_first_position(mc, D):
    """More rows than tokens: the first ones stand at negative positions, see nothing and are not read or
    written; the others are what they are without them."""
    Hkv, Hq, page = 2, 4, 16
    w = World4(mc, [20], Hkv=Hkv, D=D, page=page, seed=D)
    table = w.table.cuda()
    kv_len = torch.tensor([20], dtype=torch.int32, device="cuda")
    wide, exact = (mc.KVBatch(kv_len, table, q_start=ta.starts([n]), T=n) for n in (23, 20))
    x = w.randn(23, Hkv * D).to(BF16).cuda()
    q = w.randn(23, Hq * D).to(BF16).cuda()
    other = mc.KVCache(w.n_pages, page, Hkv, D, dtype=E2M1, k=w.cache.k.clone(), v=w.cache.v.clone())
    mc.kv_append(None, x, x, None, wide, w.cache, None)
    mc.kv_append(None, x[3:], x[3:], None, exact, other, None)
    assert torch.equal(w.cache.k, other.k) and torch.equal(w.cache.v, other.v)
    at = mc.Attention(Hq, D ** -0.5)
    sm = [mc.KVSummary(w.cache) for _ in range(2)]
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    got = []
    for i, (batch, n) in enumerate(((wide, 23), (exact, 20))):
        mc.kv_summarize(batch, w.cache, sm[i])
        k = torch.full((n, Hkv * D), 7.0, dtype=BF16, device="cuda")
        mc.kv_read(batch, w.cache, None, k)
        sel = torch.full((n, Hkv, 1), 9, dtype=torch.int32, device="cuda")
        count = torch.full((n, Hkv), 9, dtype=torch.int32, device="cuda")
        mc.attn_select(q[-n:], batch, w.cache, sm[i], at, sel, count, ws, keep_first=0)
        o, op = (torch.full((n, Hq * D), 7.0, dtype=BF16, device="cuda") for _ in range(2))
        lse, lp = (torch.full((n, Hq), 7.0, device="cuda") for _ in range(2))
        mc.attn_sparse(q[-n:], batch, w.cache, at, sel, count, o, ws, lse=lse)
        mc.attn_prefill(q[-n:], batch, w.cache, at, op, ws, lse=lp)
        got.append((k, sel, count, o, lse, op, lp))
    k, sel, count, o, lse, op, lp = got[0]
    assert bool((k[:3] == 7.0).all()) and bool((sel[:3] == -1).all()) and bool((count[:3] == 0).all())
    for x in (o, op):
        assert bool((x[:3] == 0.0).all())
    for x in (lse, lp):
        assert bool((x[:3] == float("-inf")).all())
    for a, b in zip(*got):
        assert torch.equal(a[3:], b)
    assert torch.equal(sm[0].bounds, sm[1].bounds) and torch.equal(sm[0].scale, sm[1].scale)
