"""The paged cache, attention over it and token importance without a map, on the
GPU, against the 64-bit oracle.  Every place of the cache that no sequence
holds is NaN; tolerances are the oracle's bounds."""
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


class World:
    """A cache with permuted pages, its sequences' keys and values in 64 bits, and
    NaN everywhere else."""

    def __init__(self, mc, lens, Hkv=2, D=128, page=16, dtype=BF16, seed=0, gap=0, extra_pages=2, odd=()):
        g = torch.Generator().manual_seed(seed)
        self.gen, self.lens, self.Hkv, self.D, self.page, self.dtype = g, lens, Hkv, D, page, dtype
        e4 = dtype == E4M3
        self.U = oa.unit(e4)
        used = [-(-n // page) for n in lens]
        n_pages = sum(used) + extra_pages
        order = torch.randperm(n_pages, generator=g).to(torch.int32)
        max_pages = max(1, max(used)) + gap
        self.table = torch.full((len(lens), max_pages), -7, dtype=torch.int32)
        at = 0
        for s, u in enumerate(used):
            self.table[s, :u] = order[at:at + u]
            at += u
        per = Hkv * page * D
        nan = 0x7f if e4 else 0x7fc0
        raw = torch.uint8 if e4 else torch.int16
        flats = {}
        self.scale = {"k": None, "v": None}
        for w in "kv":
            flat = torch.full((n_pages * per,), nan, dtype=raw).view(dtype)
            if e4:
                self.scale[w] = 0.01 * torch.exp(0.3 * torch.randn(Hkv, generator=g))
            for s, n in enumerate(lens):
                for h in range(Hkv):
                    x = torch.randn((n, D), generator=g)
                    if e4:
                        x = (x / self.scale[w][h]).clamp(-448, 448)
                    x = x.to(dtype)
                    for (os, oj, oh, od, ow, val) in odd:
                        if (os, oh, ow) == (s, h, w):
                            x[oj, od] = val
                    oa.write(w, flat, self.table[s], torch.arange(n), h, x, page, Hkv, D, self.U)
            flats[w] = flat
        self.flat = flats
        dev = lambda t: None if t is None else t.cuda()  # noqa: E731
        self.cache = mc.KVCache(n_pages, page, Hkv, D, dtype=dtype, k=flats["k"].view(n_pages, per).cuda(),
                                v=flats["v"].view(n_pages, per).cuda(), k_scale=dev(self.scale["k"]),
                                v_scale=dev(self.scale["v"]))

    def rows(self, w, s, h, n=None):
        r = oa.read(w, self.flat[w], self.table[s], self.lens[s] if n is None else n, h, self.page, self.Hkv, self.D,
                    self.U)
        return r if self.scale[w] is None else r * self.scale[w][h].double()

    def randn(self, *shape):
        return torch.randn(shape, generator=self.gen)

    def workspace(self, mc, T, Hq):
        return torch.full((mc.attn_workspace(T, Hq, self.Hkv, self.D),), 255, dtype=torch.uint8, device="cuda")


def starts(new):
    q = [0]
    for n in new:
        q.append(q[-1] + n)
    return torch.tensor(q, dtype=torch.int32, device="cuda")


def check(got, want, tol, what):
    got = got.double().cpu()
    bad = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[bad & ~torch.isnan(want)], want[bad & ~torch.isnan(want)]), what
    off = (got - want).abs()[~bad] - tol[~bad]
    assert off.numel() == 0 or float(off.max()) <= 0.0, "%s: %g over its bound" % (what, float(off.max()))


def run_attention(mc, w, new, Hq, decode, window=0, cap=0.0, slopes=None, prefix=None, max_len=0, lens=None,
                  wide=0, stream=None, what="", q=None):
    """Runs a call on sequences of w and compares every row with the oracle."""
    lens = w.lens if lens is None else lens
    S, D, g = len(lens), w.D, Hq // w.Hkv
    T = S if decode else sum(new)
    pad = 0 if decode else 3
    if q is None:
        q = w.randn(T + pad, Hq * D + wide).to(BF16)
    qd = q.cuda()[:, :Hq * D]
    o = torch.full((T + pad, Hq * D + wide), 7.0, dtype=BF16, device="cuda")
    lse = torch.full((T + pad, Hq), 7.0, device="cuda")
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    batch = mc.KVBatch(kv_len, w.table.cuda(), q_start=None if decode else starts(new), T=None if decode else T + pad,
                       max_len=max_len)
    at = mc.Attention(Hq, D ** -0.5, softcap=cap, window=window, slopes=None if slopes is None else slopes.cuda(),
                      prefix=None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device="cuda"))
    ws = w.workspace(mc, T + pad, Hq)
    print("%s S=%d T=%d Hq=%d lens=%s" % (what, S, T, Hq, lens[:4]), flush=True)
    (mc.attn_decode if decode else mc.attn_prefill)(qd, batch, w.cache, at, o[:, :Hq * D], ws, lse=lse, stream=stream)
    torch.cuda.synchronize()
    if wide:
        assert bool((o[:, Hq * D:] == 7.0).all()), "elements between rows were written"
    if pad:
        assert bool((o[T:] == 7.0).all()) and bool((lse[T:] == 7.0).all()), "padding rows were written"
    oc, lc = o[:T, :Hq * D].cpu().view(T, Hq, D), lse[:T].cpu()
    t0 = 0
    for s in range(S):
        n = 1 if decode else new[s]
        pos = lens[s] - n + torch.arange(n)
        for h in range(w.Hkv):
            k, v = w.rows("k", s, h, lens[s]), w.rows("v", s, h, lens[s])
            for hq in range(h * g, (h + 1) * g):
                qr = q[t0:t0 + n, hq * D:(hq + 1) * D].double()
                pre = 0 if prefix is None else min(max(0, prefix[s]), lens[s])
                ro, rl, to, tl = oa.attend(qr, k, v, pos, scale=D ** -0.5, cap=cap, window=window,
                                           slope=0.0 if slopes is None else float(slopes[hq]), prefix=pre)
                check(oc[t0:t0 + n, hq], ro, to, "%s o s=%d h=%d" % (what, s, hq))
                check(lc[t0:t0 + n, hq], rl, tl, "%s lse s=%d h=%d" % (what, s, hq))
        t0 += n
    return o, lse


# ------------------------------------------------------------------ append --

@pytest.mark.parametrize("D,Hq,Hkv,page,dtype,norm,rot,pairs", [
    (128, 4, 2, 16, BF16, "none", 128, False),
    (64, 6, 2, 32, BF16, "head", 64, True),
    (128, 3, 3, 64, BF16, "row", 128, False),
    (128, 8, 2, 16, E4M3, "head", 64, False),
    (64, 16, 16, 256, E4M3, "row", 32, True),
    (64, 1, 1, 128, BF16, "none", 0, False),
    (128, 40, 8, 16, BF16, "row", 16, False),
    (128, 96, 4, 32, E4M3, "head", 128, False),
])
def test_append(mc, D, Hq, Hkv, page, dtype, norm, rot, pairs):
    new = [1, 0, 37, 16, 5, 64, 1, 8]
    lens = [1, 9, 40, 32, 260, 64, 130, 15]
    w = World(mc, lens, Hkv=Hkv, D=D, page=page, dtype=dtype, seed=D + Hq)
    T = sum(new)
    qkv = w.randn(T + 2, (Hq + 2 * Hkv) * D).to(BF16)
    rope = torch.stack((torch.cos(w.randn(300, max(rot // 2, 1))), torch.sin(w.randn(300, max(rot // 2, 1)))), -1)
    width = {"none": 0, "head": D, "row": -1}[norm]
    wq, wk = ((1 + 0.2 * w.randn(h * D if width < 0 else D)).to(BF16) if width else None for h in (Hq, Hkv))
    prep = mc.QKPrep(rope=rope.cuda() if rot else None, rope_pairs=pairs,
                     q_norm=None if wq is None else wq.cuda(), k_norm=None if wk is None else wk.cuda(),
                     norm_row=norm == "row", eps=1e-6)
    batch = mc.KVBatch(torch.tensor(lens, dtype=torch.int32, device="cuda"), w.table.cuda(), q_start=starts(new),
                       T=T + 2)
    d = qkv.cuda()
    out = torch.full((T + 2, Hq * D + 8), 7.0, dtype=BF16, device="cuda")
    print("append", D, Hq, Hkv, page, dtype, norm, flush=True)
    mc.kv_append(d[:, :Hq * D], d[:, Hq * D:(Hq + Hkv) * D], d[:, (Hq + Hkv) * D:], prep, batch, w.cache,
                 out[:, :Hq * D])
    torch.cuda.synchronize()
    assert bool((out[T:] == 7.0).all()) and bool((out[:, Hq * D:] == 7.0).all())
    got = {x: getattr(w.cache, x).cpu().reshape(-1) for x in "kv"}
    t0 = 0
    touched = {x: torch.zeros(w.flat[x].numel(), dtype=torch.bool) for x in "kv"}
    for s, n in enumerate(new):
        pos = lens[s] - n + torch.arange(n)
        x = qkv[t0:t0 + n].double()
        args = (norm, 1e-6, rot, pairs, rope[pos].double())
        yq, eq = oa.prepare(x[:, :Hq * D], Hq, D, None if wq is None else wq.double(), *args)
        yk, ek = oa.prepare(x[:, Hq * D:(Hq + Hkv) * D], Hkv, D, None if wk is None else wk.double(), *args)
        yv = x[:, (Hq + Hkv) * D:].view(n, Hkv, D)
        check(out[t0:t0 + n, :Hq * D].cpu().view(n, Hq, D), yq, oa.BF * (yq.abs() + eq) + eq, "q_out s=%d" % s)
        for which, y, e in (("k", yk, ek), ("v", yv, torch.zeros_like(yv))):
            for h in range(Hkv):
                rows = oa._offsets(which, w.table[s], pos, h, page, Hkv, D, w.U)
                touched[which][rows.reshape(-1)] = True
                raw = torch.uint8 if dtype == E4M3 else torch.int16
                val = got[which].view(raw)[rows.reshape(-1)].view(dtype).double().view(n, D)
                yy, ee = y[:, h], e[:, h]
                if dtype == E4M3:
                    # half a step of a normal value, or of the subnormals' 2^-9; the division adds a rounding
                    sc = w.scale[which][h].double()
                    yy, ee = (yy / sc).clamp(-448, 448), ee / sc + 2 * oa.U24 * (yy / sc).abs()
                    tol = torch.clamp(2.0 ** -4 * (yy.abs() + ee), min=2.0 ** -10) + ee
                else:
                    tol = oa.BF * (yy.abs() + ee) + ee if which == "k" and (norm != "none" or rot) else 0 * yy
                check(val, yy, tol, "%s s=%d h=%d" % (which, s, h))
        t0 += n
    for x in "kv":     # everything else is as it was
        raw = torch.uint8 if dtype == E4M3 else torch.int16
        a, b = got[x].view(raw), w.flat[x].view(raw)
        assert torch.equal(a[~touched[x]], b[~touched[x]]), x


def test_append_e4m3_codes(mc):
    """Codes of every bf16 value at a power-of-two scale are the nearest ones, ties
    to even, clamped; NaN stays NaN."""
    D, page = 64, 16
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(BF16).view(-1, D)
    T = bits.shape[0]
    n_pages = T // page
    sc = torch.tensor([0.25], device="cuda")
    cache = mc.KVCache(n_pages, page, 1, D, dtype=E4M3, k_scale=sc, v_scale=sc)
    batch = mc.KVBatch(torch.tensor([T], dtype=torch.int32, device="cuda"),
                       torch.arange(n_pages, dtype=torch.int32, device="cuda").view(1, -1),
                       q_start=starts([T]), T=T)
    mc.kv_append(None, bits.cuda(), bits.cuda(), None, batch, cache, None)
    torch.cuda.synchronize()
    want = (bits.float() * 4).clamp(-448, 448).to(E4M3)          # a NaN passes through clamp
    for which in "kv":
        flat = getattr(cache, which).cpu().reshape(-1)
        at = oa._offsets(which, torch.arange(n_pages), torch.arange(T), 0, page, 1, D, 16)
        got = flat.view(torch.uint8)[at.reshape(-1)].view(E4M3).view(T, D)
        nan = torch.isnan(bits.float())
        assert torch.equal(torch.isnan(got.float()), nan)
        assert torch.equal(got.float()[~nan], want.float()[~nan]), which


def test_append_skips(mc):
    """Tokens whose position, table entry or rotation row is out of range, and rows
    outside the sequences, leave everything as it was; q_out may be q."""
    D, page, Hq, Hkv = 64, 16, 2, 1
    w = World(mc, [20, 20, 20], Hkv=Hkv, D=D, page=page, seed=3)
    table = w.table.clone()
    table[0, 1] = w.cache.n_pages           # tokens 16.. of sequence 0: no such page
    table[1, 1] = -1
    rope = torch.ones((18, D // 2, 2), device="cuda")
    rope[..., 1] = 0.0                      # the identity
    new = [6, 6, 6]                         # positions 14 .. 19
    q_start = torch.tensor([2, 8, 14, 20], dtype=torch.int32, device="cuda")
    T = 23
    x = w.randn(T, (Hq + 2 * Hkv) * D).to(BF16)
    d = x.cuda()
    batch = mc.KVBatch(torch.tensor([20, 20, 20], dtype=torch.int32, device="cuda"), table.cuda(), q_start=q_start,
                       T=T)
    scaled = torch.full((D,), 2.0, dtype=BF16, device="cuda")
    mc.kv_append(d[:, :Hq * D], d[:, Hq * D:(Hq + 1) * D], d[:, (Hq + 1) * D:],
                 mc.QKPrep(rope=rope, q_norm=scaled, k_norm=scaled, eps=0.0), batch, w.cache, d[:, :Hq * D])
    torch.cuda.synchronize()
    live = [2 + i for i in (0, 1)] + [8 + i for i in (0, 1)] + [14 + i for i in range(4)]   # positions 14 .. 17
    changed = (d.cpu().view(torch.int16) != x.view(torch.int16))[:, :Hq * D].any(1)
    assert torch.nonzero(changed).flatten().tolist() == live
    assert torch.equal(d.cpu()[:, Hq * D:], x[:, Hq * D:])
    for s in range(3):
        for which, c0 in (("k", Hq), ("v", Hq + 1)):
            flat = getattr(w.cache, which).cpu().reshape(-1)
            now = oa.read(which, flat, w.table[s], 20, 0, page, Hkv, D, w.U)
            was = w.rows(which, s, 0)
            for p in range(20):
                t = 2 + 6 * s + p - 14
                if p >= 14 and t in live:
                    if which == "v":
                        assert torch.equal(now[p], x[t, c0 * D:(c0 + 1) * D].double())
                    else:
                        assert not torch.equal(now[p], was[p])
                else:
                    assert torch.equal(now[p], was[p]), (s, which, p)


# ------------------------------------------------------------------ decode --

@pytest.mark.parametrize("D,Hq,Hkv,page,dtype", [
    (128, 8, 2, 16, BF16), (64, 2, 2, 32, BF16), (128, 34, 2, 64, BF16), (64, 15, 3, 256, BF16),
    (128, 4, 1, 16, E4M3), (64, 32, 2, 128, E4M3), (128, 3, 3, 256, E4M3),
])
@pytest.mark.parametrize("max_len", [1, 0])
def test_decode(mc, D, Hq, Hkv, page, dtype, max_len):
    """Lengths from none to a few steps of every wave, split (max_len 0: the
    tables' length) and not (a hint of one token)."""
    lens = [1, 0, 2, 15, 16, 17, 31, 33, 64, 65, 127, 129, 500, 777]
    w = World(mc, lens, Hkv=Hkv, D=D, page=page, dtype=dtype, seed=Hq)
    run_attention(mc, w, None, Hq, True, max_len=max_len, wide=8, what="decode")


@pytest.mark.parametrize("window,cap,slopes,prefix", [
    (1, 0.0, False, None), (33, 0.0, False, None), (200, 15.0, True, None), (0, 5.0, False, None),
    (0, 0.0, True, None), (40, 0.0, False, [0, 1, 7, 64, 900, -3]), (2147483647, 20.0, True, [3, 3, 3, 3, 3, 3]),
])
@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_decode_masks(mc, window, cap, slopes, prefix, dtype):
    lens = [1, 40, 77, 300, 1000, 640]
    w = World(mc, lens, Hkv=2, D=64, page=32, dtype=dtype, seed=window % 97)
    sl = torch.exp2(-torch.arange(1, 7, dtype=torch.float32)) if slopes else None
    for max_len in (1, 0):
        run_attention(mc, w, None, 6, True, window=window, cap=cap, slopes=sl, prefix=prefix, max_len=max_len,
                      what="decode masks")


def test_decode_hides_what_it_masks(mc):
    """NaN and infinities in keys and values that the window hides change nothing;
    visible ones count."""
    odd = [(0, 3, 0, 5, "v", math.nan), (0, 4, 0, 6, "v", math.inf), (0, 5, 1, 0, "k", math.nan),
           (1, 60, 1, 9, "v", math.inf), (1, 61, 1, 9, "v", -math.inf), (2, 70, 0, 1, "v", -math.inf)]
    w = World(mc, [64, 64, 90], Hkv=2, D=64, seed=5, odd=odd)
    run_attention(mc, w, None, 4, True, window=32, what="decode odd")


def test_decode_many_splits(mc):
    """One head over many parts (the most there are) and as few rows as can be."""
    w = World(mc, [40000], Hkv=1, D=64, page=256, seed=8)
    run_attention(mc, w, None, 1, True, what="decode long")
    w = World(mc, [30000, 100], Hkv=1, D=128, page=256, dtype=E4M3, seed=9)
    run_attention(mc, w, None, 16, True, what="decode long e4m3")


# ----------------------------------------------------------------- prefill --

@pytest.mark.parametrize("D,Hq,Hkv,page,dtype", [
    (128, 8, 2, 16, BF16), (64, 2, 2, 32, BF16), (128, 5, 1, 64, BF16), (64, 6, 2, 256, BF16),
    (128, 4, 4, 16, E4M3), (64, 16, 2, 128, E4M3),
])
@pytest.mark.parametrize("max_len", [1, 0])
def test_prefill(mc, D, Hq, Hkv, page, dtype, max_len):
    """Prompts and chunks over a cache, some empty, some of one token, lengths
    around the tiles' edges."""
    new = [1, 0, 7, 63, 64, 65, 1, 130, 300]
    lens = [1, 5, 7, 63, 200, 65, 513, 140, 300]
    w = World(mc, lens, Hkv=Hkv, D=D, page=page, dtype=dtype, seed=Hq)
    run_attention(mc, w, new, Hq, False, max_len=max_len, wide=8, what="prefill")


@pytest.mark.parametrize("window,cap,slopes,prefix", [
    (1, 0.0, False, None), (33, 0.0, False, None), (200, 15.0, True, None), (0, 5.0, False, None),
    (0, 0.0, True, None), (40, 0.0, False, [0, 1, 7, 64, 900, -3]), (2147483647, 20.0, True, [3, 3, 3, 3, 3, 3]),
    (0, 0.0, False, [1, 100, 300, 65, 200, 20]),
])
@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_prefill_masks(mc, window, cap, slopes, prefix, dtype):
    lens = [1, 40, 77, 300, 700, 640]
    new = [1, 40, 30, 300, 150, 3]
    w = World(mc, lens, Hkv=2, D=128, page=32, dtype=dtype, seed=window % 97)
    sl = torch.exp2(-torch.arange(1, 7, dtype=torch.float32)) if slopes else None
    for max_len in (1, 0):
        run_attention(mc, w, new, 6, False, window=window, cap=cap, slopes=sl, prefix=prefix, max_len=max_len,
                      what="prefill masks")


@pytest.mark.parametrize("D,dtype", [(64, BF16), (128, BF16), (128, E4M3)])
def test_prefill_hides_what_it_masks(mc, D, dtype):
    """A value that is not finite reaches the rows that see it and no others, in
    tiles on the diagonal, at the window's edge and inside."""
    inf = math.nan if dtype == E4M3 else math.inf
    odd = [(0, 3, 0, 5, "v", math.nan), (0, 40, 0, 6, "v", inf), (0, 41, 0, 6, "v", -inf), (0, 90, 1, 33, "v", -inf),
           (0, 91, 1, 33, "v", -inf), (0, 100, 1, 20, "v", inf), (1, 129, 0, 0, "v", inf), (1, 10, 1, 63, "v", math.nan),
           (1, 128, 1, 3, "k", math.nan)]
    w = World(mc, [140, 130], Hkv=2, D=D, dtype=dtype, seed=5, odd=odd)
    for window in (0, 30):
        run_attention(mc, w, [140, 100], 4, False, window=window, what="prefill odd")


@pytest.mark.parametrize("D,dtype", [(64, BF16), (64, E4M3), (128, BF16), (128, E4M3)])
@pytest.mark.parametrize("max_len,window", [(1, 0), (512, 0), (1, 5000), (0, 0)])
def test_prefill_long(mc, D, dtype, max_len, window):
    """More than 64 and more than 128 tiles of keys for one workgroup, of two sequences."""
    lens, new = [9001, 4160], [33, 1]
    w = World(mc, lens, Hkv=1, D=D, page=16, dtype=dtype, seed=D)
    run_attention(mc, w, new, 2, False, window=window, max_len=max_len, what="prefill long")


@pytest.mark.parametrize("window,cap,slopes,prefix", [
    (0, 0.0, False, None), (390, 0.0, False, None), (400, 15.0, True, None), (0, 5.0, False, None),
    (0, 0.0, True, None), (40, 0.0, False, [0, 1, 7, 64, 900, -3, 5]),
])
@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_prefill_by_teams(mc, window, cap, slopes, prefix, dtype):
    """Heads of 64 whose lengths are said to be long and that are not split over the keys
    (512 is one part's): halves of the keys go to two teams, one of which may have none."""
    lens = [1, 40, 77, 300, 700, 640, 0]
    new = [1, 40, 30, 300, 150, 3, 2]
    w = World(mc, lens, Hkv=2, D=64, page=32, dtype=dtype, seed=window)
    sl = torch.exp2(-torch.arange(1, 7, dtype=torch.float32)) if slopes else None
    run_attention(mc, w, new, 6, False, window=window, cap=cap, slopes=sl, prefix=prefix, max_len=512, wide=8,
                  what="prefill by teams")


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_prefill_by_teams_hides_what_it_masks(mc, dtype):
    inf = math.nan if dtype == E4M3 else math.inf
    odd = [(0, 3, 0, 5, "v", math.nan), (0, 40, 0, 6, "v", inf), (0, 41, 0, 6, "v", -inf), (0, 90, 1, 33, "v", -inf),
           (0, 100, 1, 20, "v", inf), (1, 129, 0, 0, "v", inf), (1, 10, 1, 63, "v", math.nan), (1, 128, 1, 3, "k", math.nan)]
    w = World(mc, [140, 130], Hkv=2, D=64, dtype=dtype, seed=6, odd=odd)
    for window in (0, 30):
        run_attention(mc, w, [140, 100], 4, False, window=window, max_len=512, what="prefill by teams, odd")


def test_rows_without_keys(mc):
    """More new tokens than the cache holds: rows at negative positions see no key,
    with a prefix too; scores of -infinity alone give no weight either."""
    w = World(mc, [3, 0, 50], Hkv=1, D=64, seed=6)
    kv = w.lens
    q = w.randn(3 + 78, 2 * 64).to(BF16)
    for prefix in (None, [3, 3, 3]):
        run_attention(mc, w, [10, 8, 60], 2, False, prefix=prefix, what="no keys", lens=kv, q=q)
    # one dimension at the type's largest values: every score overflows to -infinity
    odd = [(0, j, 0, 0, "k", -3e38) for j in range(5)]
    w = World(mc, [5], Hkv=1, D=64, seed=6, odd=odd)
    q = torch.zeros((1, 64), dtype=BF16)
    q[0, 0] = 3e38
    o = torch.empty((1, 64), dtype=BF16, device="cuda")
    lse = torch.empty((1, 1), device="cuda")
    for call, kw in ((mc.attn_decode, {}), (mc.attn_prefill, dict(q_start=starts([1]), T=1))):
        batch = mc.KVBatch(torch.tensor([5], dtype=torch.int32, device="cuda"), w.table.cuda(), **kw)
        call(q.cuda(), batch, w.cache, mc.Attention(1, 1.0), o, w.workspace(mc, 1, 1), lse=lse)
        torch.cuda.synchronize()
        assert bool((o == 0).all()) and float(lse) == -math.inf


# -------------------------------------------------------------- importance --

@pytest.mark.parametrize("D,Hq,Hkv,page,dtype,L,d,window,cap,slopes", [
    (128, 8, 2, 16, BF16, 1, 64, 0, 0.0, False), (128, 8, 2, 16, BF16, 300, 129, 0, 0.0, False),
    (64, 4, 4, 64, BF16, 513, 256, 0, 0.0, False), (128, 6, 2, 256, E4M3, 290, 64, 0, 0.0, False),
    (64, 3, 1, 32, E4M3, 257, 40, 0, 0.0, False), (64, 4, 2, 16, BF16, 400, 64, 33, 20.0, True),
    (128, 2, 2, 128, BF16, 600, 64, 300, 0.0, False), (128, 16, 1, 16, E4M3, 64, 64, 1, 0.0, True),
])
def test_importance(mc, D, Hq, Hkv, page, dtype, L, d, window, cap, slopes):
    w = World(mc, [L], Hkv=Hkv, D=D, page=page, dtype=dtype, seed=L)
    sl = torch.exp2(-torch.arange(1, Hq + 1, dtype=torch.float32)) if slopes else None
    q = (w.randn(L + 3, Hq * D)).to(BF16)
    _, lse = run_attention(mc, w, [L], Hq, False, window=window, cap=cap, slopes=sl, q=q, what="importance")
    x = w.randn(L, d).to(BF16)
    batch = mc.KVBatch(torch.tensor([L], dtype=torch.int32, device="cuda"), w.table.cuda(), q_start=starts([L]), T=L)
    at = mc.Attention(Hq, D ** -0.5, softcap=cap, window=window, slopes=None if sl is None else sl.cuda())
    imp = torch.full((L,), -1.0, device="cuda")
    mask = torch.full((L,), 9, dtype=torch.uint8, device="cuda")
    ws = torch.full((mc.attn_importance_workspace(Hq, L),), 255, dtype=torch.uint8, device="cuda")
    lse = lse[:L].contiguous()
    for rho in (0.1, 0.0, 1.0):
        mc.attn_importance(q[:L].cuda(), lse, batch, w.cache, at, x.cuda(), rho, mask, ws, importance=imp)
        torch.cuda.synchronize()
        want, rel = oa.importance(q[:L].double(), lse.double().cpu(), [w.rows("k", 0, h) for h in range(Hkv)],
                                  x.double(), L, Hq // Hkv, Hkv, D, scale=D ** -0.5, cap=cap, window=window,
                                  slopes=sl)
        check(imp, want, rel * want, "importance")
        n = int(math.floor(float(torch.tensor(rho, dtype=torch.float32)) * L + 0.5))
        order = torch.sort(imp.cpu(), descending=True, stable=True).indices
        top = torch.zeros(L, dtype=torch.uint8)
        top[order[:n]] = 1
        assert torch.equal(mask.cpu(), top), rho
