"""The cache and attention calls as a program uses them: prompts and decode steps of a
decoder block with its MoE layer, captured and replayed graphs, streams, caches that
share an allocation, offsets beyond 32 bits, the same call twice."""
import math

import pytest

torch = pytest.importorskip("torch")

from oracle import attention as oa  # noqa: E402

pytestmark = pytest.mark.gpu

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def mc():
    import paper_2410_06270_amd as m
    m.load()
    return m


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rope_table(n, rot, base=10000.0):
    at = torch.arange(n, dtype=torch.float64)[:, None]
    ang = at * base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.stack((ang.cos(), ang.sin()), -1).float().contiguous()


class Heads:
    """One layer's attention: projections' outputs in, attention out, by the calls."""

    def __init__(self, mc, lens, Hq, Hkv, D, page=16, dtype=BF16, seed=0, **attn):
        self.mc, self.Hq, self.Hkv, self.D, self.page = mc, Hq, Hkv, D, page
        self.gen = torch.Generator().manual_seed(seed)
        self.max_pages = max(-(-n // page) for n in lens)
        S = len(lens)
        n_pages = S * self.max_pages
        self.table = torch.randperm(n_pages, generator=self.gen).to(torch.int32).view(S, -1).cuda()
        sc = torch.full((Hkv,), 0.02, device="cuda") if dtype == E4M3 else None
        self.cache = mc.KVCache(n_pages, page, Hkv, D, dtype=dtype, k_scale=sc, v_scale=sc)
        w = (1 + 0.1 * torch.randn(D, generator=self.gen)).to(BF16).cuda()
        self.prep = mc.QKPrep(rope=rope_table(max(lens) + 1, D).cuda(), q_norm=w, k_norm=w, eps=1e-5)
        self.attn = mc.Attention(Hq, D ** -0.5, **attn)

    def batch(self, lens, new):
        q = [0]
        for n in new:
            q.append(q[-1] + n)
        return self.mc.KVBatch(i32(lens), self.table, q_start=i32(q), T=q[-1], max_len=max(lens))

    def append(self, qkv, batch, q_out):
        a, b = self.Hq * self.D, (self.Hq + self.Hkv) * self.D
        self.mc.kv_append(qkv[:, :a], qkv[:, a:b], qkv[:, b:], self.prep, batch, self.cache, q_out)

    def workspace(self, T):
        return torch.empty(self.mc.attn_workspace(T, self.Hq, self.Hkv, self.D), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_decode_continues_prefill(mc, dtype):
    """Prompts in one call, then tokens one by one, agree with all tokens in one call:
    the two read the same cache, so they differ only by the weights' rounding to bf16
    and fp32 sums, 2^-8 sum w |v| a side and a rounding of the result each."""
    lens, steps = [37, 5, 64], 4
    total = [n + steps for n in lens]
    h = Heads(mc, total, 8, 2, 64, dtype=dtype, seed=1)
    qkv = [torch.randn((t, 12 * 64), generator=h.gen).to(BF16).cuda() for t in total]
    # all at once
    every = torch.cat(qkv)
    T = every.shape[0]
    b = h.batch(total, total)
    q_all = torch.empty((T, 8 * 64), dtype=BF16, device="cuda")
    h.append(every, b, q_all)
    o_all, lse_all = torch.empty_like(q_all), torch.empty((T, 8), device="cuda")
    mc.attn_prefill(q_all, b, h.cache, h.attn, o_all, h.workspace(T), lse=lse_all)
    torch.cuda.synchronize()
    k_all, v_all = h.cache.k.clone(), h.cache.v.clone()
    absv = float(v_all.float().abs().max()) * (0.02 if dtype == E4M3 else 1.0)
    h.cache.k.view(torch.uint8).zero_()
    h.cache.v.view(torch.uint8).zero_()
    # prompts, then steps
    first = torch.cat([x[:n] for x, n in zip(qkv, lens)])
    b = h.batch(lens, lens)
    q1 = torch.empty((first.shape[0], 8 * 64), dtype=BF16, device="cuda")
    h.append(first, b, q1)
    o1 = torch.empty_like(q1)
    mc.attn_prefill(q1, b, h.cache, h.attn, o1, h.workspace(first.shape[0]))
    starts = [0, total[0], total[0] + total[1]]
    # (and lse by the fp32 products: 70 2^-24 sum |q k| / 8 <= 4e-5 a side after the norms)
    tol = 2 * (2.0 ** -8 * absv + 2.0 ** -8 * absv)
    for i in range(steps):
        now = [n + i + 1 for n in lens]
        b = h.batch(now, [1] * 3)
        row = torch.cat([x[n - 1:n] for x, n in zip(qkv, now)])
        q, o, lse = torch.empty((3, 512), dtype=BF16, device="cuda"), torch.empty((3, 512), dtype=BF16, device="cuda"), \
            torch.empty((3, 8), device="cuda")
        h.append(row, b, q)
        mc.attn_decode(q, b, h.cache, h.attn, o, h.workspace(3), lse=lse)
        torch.cuda.synchronize()
        at = [s + n - 1 for s, n in zip(starts, now)]
        assert torch.equal(q, q_all[at])
        assert float((o.float() - o_all[at].float()).abs().max()) <= tol
        assert float((lse - lse_all[at]).abs().max()) <= 1e-4
    assert torch.equal(h.cache.k.view(torch.uint8), k_all.view(torch.uint8))
    assert torch.equal(h.cache.v.view(torch.uint8), v_all.view(torch.uint8))
    t0 = 0
    for s, n in zip(starts, lens):
        assert float((o1[t0:t0 + n].float() - o_all[s:s + n].float()).abs().max()) <= tol
        t0 += n


def test_block_with_moe(mc):
    """A prompt through append, prefill, importance, routing with the protected tokens
    and the packed experts: the mask is what mc_token_importance gives for the map of
    the same scores (its bf16 rounding aside), and the layer runs on it."""
    Hq, Hkv, D, L, d = 4, 2, 64, 200, 256
    h = Heads(mc, [L], Hq, Hkv, D, seed=2)
    qkv = (2 * torch.randn((L, (Hq + 2 * Hkv) * D), generator=h.gen)).to(BF16).cuda()
    b = h.batch([L], [L])
    q = torch.empty((L, Hq * D), dtype=BF16, device="cuda")
    h.append(qkv, b, q)
    o, lse = torch.empty_like(q), torch.empty((L, Hq), device="cuda")
    mc.attn_prefill(q, b, h.cache, h.attn, o, h.workspace(L), lse=lse)
    x = o.contiguous()                                   # the MoE layer's input
    rho = 0.1
    imp, mask = torch.empty(L, device="cuda"), torch.empty(L, dtype=torch.uint8, device="cuda")
    ws = torch.empty(mc.attn_importance_workspace(Hq, L), dtype=torch.uint8, device="cuda")
    mc.attn_importance(q, lse, b, h.cache, h.attn, x, rho, mask, ws, importance=imp)
    torch.cuda.synchronize()
    # the map by the oracle, in bf16, through mc_token_importance
    flat = h.cache.k.cpu().reshape(-1)
    maps = torch.zeros((Hq, L, L), dtype=torch.float64)
    for hq in range(Hq):
        k = oa.read("k", flat, h.table[0].cpu(), L, hq // 2, h.page, Hkv, D, 8)
        s, _ = oa.scores(q.cpu()[:, hq * D:(hq + 1) * D].double(), k, torch.arange(L), scale=D ** -0.5)
        maps[hq] = torch.exp(s - lse.cpu()[:, hq:hq + 1].double())
    amap = maps.to(BF16).cuda()
    imp2, mask2 = torch.empty_like(imp), torch.empty_like(mask)
    ws2 = torch.empty(mc.importance_workspace(Hq, L), dtype=torch.uint8, device="cuda")
    mc.token_importance(amap.view(torch.int16), x.view(torch.int16), rho, mask2, ws2, importance=imp2)
    torch.cuda.synchronize()
    # every probability of the map is off by 2^-8 of itself at most
    assert bool(((imp - imp2).abs() <= (2.0 ** -8 + 1e-4) * imp2).all())
    cut = torch.sort(imp2, descending=True).values[int(rho * L) - 1]
    apart = (imp2 - cut).abs() > 2 * 2.0 ** -8 * cut + 1e-6
    assert torch.equal(mask[apart], mask2[apart]) and int(mask.sum()) == int(mask2.sum()) == 20
    # the MoE layer with the mask
    E, ffn, k = 4, 512, 2
    w = [torch.randn((E, ffn, d) if m < 2 else (E, d, ffn), generator=h.gen).mul_(0.02).cuda() for m in range(3)]
    layer = mc.PackedLayer(E, d, ffn, [3, 2, 1, 2], 32)
    mc.pack(*w, layer)
    wr = torch.randn((E, d), generator=h.gen).to(BF16).cuda()
    logits = torch.empty((L, E), device="cuda")
    xi = x.view(torch.int16)
    mc.router_logits(xi, wr.view(torch.int16), logits)
    r = mc.Routing(L, E, k)
    mc.route_and_prune(logits, mask, 0.49, r)
    y = torch.empty((L, d), dtype=torch.int16, device="cuda")
    mc.moe_forward(xi, r, layer, y, torch.empty(mc.forward_workspace(L, E, k, d, ffn), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert bool((r.kept[mask.bool()] == 1).all())        # protected tokens keep both experts
    assert int(r.n_pruned) > 0
    assert bool(torch.isfinite(y.view(BF16).float()).all())


def test_graph_replays(mc):
    """A decode step captured once and replayed as the sequences grow: lengths and rows
    change in place, and every replay equals the eager call.  Two graphs share a
    workspace; eager work of its own goes between the replays."""
    lens = [50, 3, 120]
    h = Heads(mc, [n + 8 for n in lens], 8, 2, 64, seed=3)
    S = 3
    kv_len = i32(lens)
    q_start = i32([0, 1, 2, 3])
    b = mc.KVBatch(kv_len, h.table, q_start=q_start, T=S, max_len=128)
    qkv = torch.zeros((S, 12 * 64), dtype=BF16, device="cuda")
    q, o, lse = torch.empty((S, 512), dtype=BF16, device="cuda"), torch.empty((S, 512), dtype=BF16, device="cuda"), \
        torch.empty((S, 8), device="cuda")
    o2 = torch.empty_like(o)
    ws = h.workspace(S)
    prompt = torch.randn((sum(lens), 12 * 64), generator=h.gen).to(BF16).cuda()
    bp = h.batch(lens, lens)
    h.append(prompt, bp, torch.empty((sum(lens), 512), dtype=BF16, device="cuda"))
    torch.cuda.synchronize()

    def step(out):
        h.append(qkv, b, q)
        mc.attn_decode(q, b, h.cache, h.attn, out, ws, lse=lse)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        kv_len += 1
        step(o)
        kv_len -= 1
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for out in (o, o2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(out)
        graphs.append(g)
    for i in range(6):
        kv_len += 1
        qkv.copy_(torch.randn((S, 12 * 64), generator=h.gen).to(BF16))
        for g, out in zip(graphs, (o, o2)):
            out.fill_(7.0)
            lse.fill_(7.0)
            g.replay()
            torch.cuda.synchronize()
            got, got_lse = out.clone(), lse.clone()
            ws.fill_(255)                                # the workspace holds nothing between calls
            eager = torch.empty_like(out)
            step(eager)
            torch.cuda.synchronize()
            assert torch.equal(got, eager) and torch.equal(got_lse, lse), i


def test_graph_of_prefill_and_importance(mc):
    """Prefill and importance captured together and replayed on new contents."""
    Hq, Hkv, D, L = 4, 2, 128, 300
    h = Heads(mc, [L], Hq, Hkv, D, page=32, seed=4)
    b = h.batch([L], [L])
    qkv = torch.randn((L, 8 * D), generator=h.gen).to(BF16).cuda()
    q = torch.empty((L, Hq * D), dtype=BF16, device="cuda")
    o, lse = torch.empty_like(q), torch.empty((L, Hq), device="cuda")
    x = torch.randn((L, 64), generator=h.gen).to(BF16).cuda()
    imp, mask = torch.empty(L, device="cuda"), torch.empty(L, dtype=torch.uint8, device="cuda")
    ws, wi = h.workspace(L), torch.empty(mc.attn_importance_workspace(Hq, L), dtype=torch.uint8, device="cuda")

    def step():
        h.append(qkv, b, q)
        mc.attn_prefill(q, b, h.cache, h.attn, o, ws, lse=lse)
        mc.attn_importance(q, lse, b, h.cache, h.attn, x, 0.1, mask, wi, importance=imp)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(4):
        qkv.copy_(torch.randn((L, 8 * D), generator=h.gen).to(BF16))
        o.fill_(7.0)
        mask.fill_(9)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (o, lse, imp, mask)]
        wi.fill_(255)
        step()
        torch.cuda.synchronize()
        for a, c in zip(got, (o, lse, imp, mask)):
            assert torch.equal(a, c)


def test_streams_and_repeats(mc):
    """Calls on a stream of their own, two at once with a workspace each, and the same
    call again, give the same bits."""
    h = Heads(mc, [3000, 70], 8, 2, 128, page=64, seed=5)
    h.cache.k.copy_(torch.randn(h.cache.k.shape, generator=h.gen).to(BF16))
    h.cache.v.copy_(torch.randn(h.cache.v.shape, generator=h.gen).to(BF16))
    q = torch.randn((2, 8 * 128), generator=h.gen).to(BF16).cuda()
    b = mc.KVBatch(i32([3000, 70]), h.table, q_start=i32([0, 1, 2]), T=2)
    ref, o1, o2, o3 = (torch.empty_like(q) for _ in range(4))
    ws = [h.workspace(2) for _ in range(3)]
    mc.attn_decode(q, b, h.cache, h.attn, ref, ws[0])
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        mc.attn_decode(q, b, h.cache, h.attn, o1, ws[1], stream=s1)
        with torch.cuda.stream(s2):
            mc.attn_decode(q, b, h.cache, h.attn, o2, ws[2])
        mc.attn_decode(q, b, h.cache, h.attn, o3, ws[0])
        torch.cuda.synchronize()
        for o in (o1, o2, o3):
            assert torch.equal(o, ref)
    # prefill of one token a sequence sees what decode sees: two kernels, whose weights
    # are rounded to bf16 apart
    mc.attn_prefill(q, b, h.cache, h.attn, o1, ws[0])
    torch.cuda.synchronize()
    assert float((o1.float() - ref.float()).abs().max()) <= 4 * 2.0 ** -8 * float(h.cache.v.float().abs().max())


@pytest.mark.parametrize("which", ["decode", "prefill", "importance"])
def test_shared_allocation_and_far_offsets(mc, which):
    """Two layers' pages interleaved in one allocation, with more than 4 GiB between
    the first page and the last: each layer reads and writes its own."""
    Hq, Hkv, D, page, n_pages = 2, 2, 64, 16, 5
    per = page * Hkv * D
    stride = 600 << 20                                    # elements: 1.2 GB between pages
    big = torch.empty((n_pages - 1) * stride + 2 * per, dtype=BF16, device="cuda")
    k0 = big.as_strided((n_pages, per), (stride, 1))
    k1 = big.as_strided((n_pages, per), (stride, 1), per)
    vbig = torch.empty_like(big)
    v0 = vbig.as_strided((n_pages, per), (stride, 1))
    v1 = vbig.as_strided((n_pages, per), (stride, 1), per)
    gen = torch.Generator().manual_seed(6)
    flat = {}
    for name, t in (("k0", k0), ("v0", v0), ("k1", k1), ("v1", v1)):
        flat[name] = torch.randn((n_pages, per), generator=gen).to(BF16)
        t.copy_(flat[name].cuda())
    table = torch.tensor([[4, 0, 3, 1]], dtype=torch.int32)
    L = 60
    cache = mc.KVCache(n_pages, page, Hkv, D, k=k0, v=v0)
    assert cache.desc.page_stride == 2 * stride
    at = mc.Attention(Hq, D ** -0.5)
    T = 1 if which == "decode" else L
    b = mc.KVBatch(i32([L]), table.cuda(), q_start=i32([0, T]), T=T)
    x = torch.randn((T, 6 * D), generator=gen).to(BF16).cuda()
    q = torch.empty((T, Hq * D), dtype=BF16, device="cuda")
    mc.kv_append(x[:, :2 * D], x[:, 2 * D:4 * D], x[:, 4 * D:], None, b, cache, q)
    torch.cuda.synchronize()
    assert torch.equal(q, x[:, :2 * D])
    assert torch.equal(k1.cpu(), flat["k1"]) and torch.equal(v1.cpu(), flat["v1"])
    kf, vf = k0.cpu().reshape(-1), v0.cpu().reshape(-1)
    o, lse = torch.empty_like(q), torch.empty((T, Hq), device="cuda")
    ws = torch.empty(mc.attn_workspace(T, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    (mc.attn_decode if which == "decode" else mc.attn_prefill)(q, b, cache, at, o, ws, lse=lse)
    torch.cuda.synchronize()
    ks = []
    for h in range(Hq):
        k = oa.read("k", kf, table[0], L, h, page, Hkv, D, 8)
        v = oa.read("v", vf, table[0], L, h, page, Hkv, D, 8)
        ks.append(k)
        assert torch.equal(k[L - T:], x.cpu()[:, (2 + h) * D:(3 + h) * D].double())
        ro, rl, to, tl = oa.attend(q.cpu()[:, h * D:(h + 1) * D].double(), k, v, torch.arange(L - T, L), scale=D ** -0.5)
        assert bool(((o.cpu()[:, h * D:(h + 1) * D].double() - ro).abs() <= to).all())
        assert bool(((lse.cpu()[:, h].double() - rl).abs() <= tl).all())
    if which == "importance":
        xx = torch.randn((L, 72), generator=gen).to(BF16).cuda()
        imp, mask = torch.empty(L, device="cuda"), torch.empty(L, dtype=torch.uint8, device="cuda")
        wi = torch.empty(mc.attn_importance_workspace(Hq, L), dtype=torch.uint8, device="cuda")
        mc.attn_importance(q, lse, b, cache, at, xx, 0.5, mask, wi, importance=imp)
        torch.cuda.synchronize()
        want, rel = oa.importance(q.cpu().double(), lse.cpu().double(), ks, xx.cpu().double(), L, 1, Hkv, D,
                                  scale=D ** -0.5)
        assert bool(((imp.cpu().double() - want).abs() <= rel * want).all()) and int(mask.sum()) == 30
    del big, vbig, k0, k1, v0, v1, cache
    torch.cuda.empty_cache()


def test_tables_with_stray_entries(mc):
    """Page numbers and lengths out of range read some page of the cache and nothing
    else: the call ends, other sequences are right."""
    Hq, Hkv, D, page = 2, 1, 64, 16
    gen = torch.Generator().manual_seed(7)
    k, v = (torch.randn((6, page * D), generator=gen).to(BF16) for _ in range(2))
    cache = mc.KVCache(6, page, Hkv, D, k=k.cuda(), v=v.cuda())
    table = torch.tensor([[99, -5, 2 ** 31 - 1, -2 ** 31], [1, 5, 0, 3], [2, 2, 2, 2]], dtype=torch.int32)
    lens = [60, 50, 2 ** 31 - 1]                          # the last: cut to what the table holds
    q = torch.randn((3, Hq * D), generator=gen).to(BF16)
    at = mc.Attention(Hq, D ** -0.5)
    ws = torch.empty(mc.attn_workspace(3, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    for call, kw in ((mc.attn_decode, {}), (mc.attn_prefill, dict(q_start=i32([0, 1, 2, 3]), T=3))):
        b = mc.KVBatch(i32(lens), table.cuda(), **kw)
        o, lse = torch.empty((3, Hq * D), dtype=BF16, device="cuda"), torch.empty((3, Hq), device="cuda")
        call(q.cuda(), b, cache, at, o, ws, lse=lse)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(o.float()).all())
        for s, n in ((1, 50), (2, 64)):
            kk = oa.read("k", k.reshape(-1), table[s], n, 0, page, Hkv, D, 8)
            vv = oa.read("v", v.reshape(-1), table[s], n, 0, page, Hkv, D, 8)
            for h in range(Hq):
                ro, rl, to, tl = oa.attend(q[s:s + 1, h * D:(h + 1) * D].double(), kk, vv, [n - 1], scale=D ** -0.5)
                assert bool(((o[s, h * D:(h + 1) * D].cpu().double() - ro[0]).abs() <= to[0]).all())
                assert math.fabs(float(lse[s, h]) - float(rl)) <= float(tl)
    # starts that are not ascending, negative or beyond the rows: nothing out of the rows is touched
    for starts in ([0, 2, 1, 3], [-4, 1, 2, 3], [0, 1, 2, 900], [5, 5, 5, 5], [3, 2, 1, 0]):
        b = mc.KVBatch(i32(lens), table.cuda(), q_start=i32(starts), T=3)
        o = torch.zeros((3, Hq * D), dtype=BF16, device="cuda")
        mc.attn_prefill(q.cuda(), b, cache, at, o, ws)
        mc.kv_append(q.cuda(), q[:, :D].contiguous().cuda(), q[:, D:].contiguous().cuda(), None, b, cache, o)
        torch.cuda.synchronize()


def test_negative_and_zero_scale(mc):
    """Scores may be any multiple of the products."""
    Hkv, D, page, L = 1, 64, 16, 150
    gen = torch.Generator().manual_seed(8)
    k, v = (torch.randn((10, page * D), generator=gen).to(BF16) for _ in range(2))
    cache = mc.KVCache(10, page, Hkv, D, k=k.cuda(), v=v.cuda())
    table = torch.randperm(10, generator=gen).to(torch.int32).view(1, -1)
    kk = oa.read("k", k.reshape(-1), table[0], L, 0, page, Hkv, D, 8)
    vv = oa.read("v", v.reshape(-1), table[0], L, 0, page, Hkv, D, 8)
    q = torch.randn((L, 2 * D), generator=gen).to(BF16)
    ws = torch.empty(mc.attn_workspace(L, 2, Hkv, D), dtype=torch.uint8, device="cuda")
    for scale in (-0.2, 0.0, 1.5):
        for cap in (0.0, 3.0):
            at = mc.Attention(2, scale, softcap=cap)
            b = mc.KVBatch(i32([L]), table.cuda(), q_start=i32([0, L]), T=L)
            o = torch.empty((L, 2 * D), dtype=BF16, device="cuda")
            mc.attn_prefill(q.cuda(), b, cache, at, o, ws)
            od = torch.empty((1, 2 * D), dtype=BF16, device="cuda")
            mc.attn_decode(q[-1:].cuda(), b, cache, at, od, ws)
            torch.cuda.synchronize()
            for h in range(2):
                ro, _, to, _ = oa.attend(q[:, h * D:(h + 1) * D].double(), kk, vv, torch.arange(L), scale=scale, cap=cap)
                assert bool(((o.cpu()[:, h * D:(h + 1) * D].double() - ro).abs() <= to).all()), (scale, cap)
                assert bool(((od.cpu()[0, h * D:(h + 1) * D].double() - ro[-1]).abs() <= to[-1]).all()), (scale, cap)


def test_binding_refusals(mc):
    """Shapes and types that do not fit are refused before the call."""
    h = Heads(mc, [32], 2, 1, 64)
    b = h.batch([32], [2])
    q, o, ws = torch.zeros((2, 128), dtype=BF16, device="cuda"), \
        torch.zeros((2, 128), dtype=BF16, device="cuda"), h.workspace(2)
    for bad in (dict(q=q[:1]), dict(o=o[:, :64]), dict(q=q.float()), dict(q=q.cpu()), dict(lse=torch.zeros(3, device="cuda")),
                dict(q=torch.zeros((128, 2), dtype=BF16, device="cuda").t())):
        args = dict(q=q, o=o, lse=None)
        args.update(bad)
        with pytest.raises(AssertionError):
            mc.attn_prefill(args["q"], b, h.cache, h.attn, args["o"], ws, lse=args["lse"])
    with pytest.raises(mc.MCError):
        mc.attn_prefill(q, b, h.cache, h.attn, o, ws[:16])
    with pytest.raises(AssertionError):
        mc.kv_append(q, q, q, None, b, h.cache, o)          # k and v are 64 wide
    with pytest.raises(AssertionError):
        mc.KVCache(4, 16, 1, 64, dtype=E4M3)                 # no scales


def test_descriptors_on_one_gpu(mc):
    """A descriptor's tensors all lie on the device of the call, and rows are bf16."""
    h = Heads(mc, [32], 2, 1, 64)
    b = h.batch([32], [2])
    q = torch.zeros((2, 128), dtype=BF16, device="cuda")
    ws, f32 = h.workspace(2), dict(dtype=torch.float32)
    with pytest.raises(AssertionError):
        mc.attn_prefill(q.half(), b, h.cache, h.attn, q, ws)
    for bad in (dict(slopes=torch.zeros(2, **f32)), dict(prefix=torch.zeros(1, dtype=torch.int32)),
                dict(slopes=torch.zeros(2, device="cuda", **f32), prefix=torch.zeros(1, dtype=torch.int32))):
        with pytest.raises(AssertionError):
            mc.Attention(2, 1.0, **bad)
    with pytest.raises(AssertionError):
        mc.KVBatch(i32([32]), h.table.cpu())
    with pytest.raises(AssertionError):
        mc.KVBatch(i32([32]), h.table, q_start=torch.tensor([0, 2], dtype=torch.int32), T=2)
    with pytest.raises(AssertionError):
        mc.QKPrep(rope=rope_table(4, 64))
    with pytest.raises(AssertionError):
        mc.KVCache(2, 16, 1, 64, dtype=E4M3, k_scale=torch.ones(1), v_scale=torch.ones(1, device="cuda"))
    with pytest.raises(AssertionError):
        mc.KVCache(2, 16, 1, 64, k=torch.zeros((2, 1024), dtype=torch.float16, device="cuda"))


@pytest.mark.parametrize("window", [500, 1 << 30, (1 << 31) - 1])
def test_windows_of_everything(mc, window):
    """A window that hides nothing, up to the largest there is, gives what no window gives
    (of 500 tokens: but for rounding, as the work may be split otherwise)."""
    L, Hq, Hkv, D = 333, 4, 2, 64
    outs = []
    for w in (0, window):
        h = Heads(mc, [L], Hq, Hkv, D, seed=3, window=w)
        qkv = torch.randn((L, (Hq + 2 * Hkv) * D), generator=torch.Generator().manual_seed(4)).to(BF16).cuda()
        q, o = (torch.empty((L, Hq * D), dtype=BF16, device="cuda") for _ in range(2))
        od = torch.empty((1, Hq * D), dtype=BF16, device="cuda")
        lse, imp = torch.empty((L, Hq), device="cuda"), torch.empty(L, device="cuda")
        mask, b = torch.empty(L, dtype=torch.uint8, device="cuda"), h.batch([L], [L])
        h.append(qkv, b, q)
        mc.attn_prefill(q, b, h.cache, h.attn, o, h.workspace(L), lse=lse)
        mc.attn_decode(q[-1:], b, h.cache, h.attn, od, h.workspace(1))
        x = torch.ones((L, 64), dtype=BF16, device="cuda")
        ws = torch.empty(mc.attn_importance_workspace(Hq, L), dtype=torch.uint8, device="cuda")
        mc.attn_importance(q, lse, b, h.cache, h.attn, x, 0.1, mask, ws, importance=imp)
        torch.cuda.synchronize()
        outs.append([t.cpu() for t in (o, od, lse, imp, mask)])
    if window >= 1 << 30:
        assert all(torch.equal(x, y) for x, y in zip(*outs))
    else:
        # on either side the weights' rounding and the output's, each 2^-8 of the largest value
        far = 4 * 2.0 ** -8 * float(qkv[:, -Hkv * D:].abs().max())
        for x, y, tol in zip(outs[0], outs[1], (far, far, 1e-5)):
            assert bool(((x.double() - y.double()).abs() <= tol).all())


def test_capped_products_past_fp32(mc):
    """A product that overflows fp32 scores at the cap, below as above, in tiles that
    every row sees and in masked ones, and hidden keys stay hidden."""
    D, page, L, cap = 64, 16, 200, 4.0
    gen = torch.Generator().manual_seed(12)
    k, v = (torch.randn((13, page * D), generator=gen).to(BF16) for _ in range(2))
    table = torch.arange(13, dtype=torch.int32).view(1, -1)
    flat = k.view(-1)
    for pos, sign in ((3, 1.0), (20, -1.0), (100, -1.0), (150, 1.0), (190, -1.0), (199, -1.0)):
        for i in range(D):
            flat[oa.offset("k", pos // page, 0, pos % page, i, page, 1, D, 8)] = sign * 2.0 ** 126
    kk = oa.read("k", flat, table[0], L, 0, page, 1, D, 8)
    vv = oa.read("v", v.reshape(-1), table[0], L, 0, page, 1, D, 8)
    q = (4 + torch.rand((L, D), generator=gen)).to(BF16)
    cache = mc.KVCache(13, page, 1, D, k=k.cuda(), v=v.cuda())
    at = mc.Attention(1, 1.0, softcap=cap)
    b = mc.KVBatch(i32([L]), table.cuda(), q_start=i32([0, L]), T=L)
    o, od = (torch.empty((n, D), dtype=BF16, device="cuda") for n in (L, 1))
    ws = torch.empty(mc.attn_workspace(L, 1, 1, D), dtype=torch.uint8, device="cuda")
    mc.attn_prefill(q.cuda(), b, cache, at, o, ws)
    mc.attn_decode(q[-1:].cuda(), b, cache, at, od, ws)
    torch.cuda.synchronize()
    ro, _, _, _ = oa.attend(q.double(), kk, vv, torch.arange(L), scale=1.0, cap=cap)
    # the weights' rounding and the output's, 2^-8 of the largest value each; the scores,
    # of which a product past 100 caps moves none, add less than a third such part
    tol = 3 * 2.0 ** -8 * float(v.float().abs().max())
    assert bool(((o.cpu().double() - ro).abs() <= tol).all())
    assert bool(((od.cpu().double() - ro[-1:]).abs() <= tol).all())


@pytest.mark.parametrize("cap", [1e-30, 1e-42])
def test_smallest_caps(mc, cap):
    """Scores within a cap that is next to nothing are next to nothing, a product of 0
    among them: every row is the mean of the values it sees."""
    D, page, L = 64, 16, 100
    gen = torch.Generator().manual_seed(13)
    k, v = (torch.randn((7, page * D), generator=gen).to(BF16) for _ in range(2))
    vv = oa.read("v", v.reshape(-1), torch.arange(7, dtype=torch.int32), L, 0, page, 1, D, 8)
    q = torch.randn((L, D), generator=gen).to(BF16)
    q[50] = 0
    q[-1] = 0
    cache = mc.KVCache(7, page, 1, D, k=k.cuda(), v=v.cuda())
    at = mc.Attention(1, 1.0, softcap=cap)
    b = mc.KVBatch(i32([L]), torch.arange(7, dtype=torch.int32).view(1, -1).cuda(), q_start=i32([0, L]), T=L)
    o, od = (torch.empty((n, D), dtype=BF16, device="cuda") for n in (L, 1))
    lse = torch.empty((L, 1), device="cuda")
    ws = torch.empty(mc.attn_workspace(L, 1, 1, D), dtype=torch.uint8, device="cuda")
    mc.attn_prefill(q.cuda(), b, cache, at, o, ws, lse=lse)
    mc.attn_decode(q[-1:].cuda(), b, cache, at, od, ws)
    torch.cuda.synchronize()
    n = torch.arange(1, L + 1, dtype=torch.float64)[:, None]
    want = vv.cumsum(0) / n
    # weights of 1 are exact in bf16: the sums (100 terms) and the output's rounding
    tol = 2.0 ** -8 * want.abs() + 200 * 2.0 ** -24 * vv.abs().amax()
    assert bool(((o.cpu().double() - want).abs() <= tol).all())
    assert bool(((od.cpu().double() - want[-1:]).abs() <= tol[-1:]).all())
    # exp, sum and logarithm in fp32: some roundings of a value below 5
    assert bool(((lse.cpu().double() - n.log()).abs() <= 8 * 2.0 ** -24 * 5).all())
