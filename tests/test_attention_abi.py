"""Refusals of the cache and attention calls: every bad argument is turned down on the
host (these calls return before any HIP call, so they run without a GPU), and the
oracle's layout is the header's."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

from oracle import attention as oa  # noqa: E402

EINVAL, ENOSPACE, EUNSUPPORTED = 1, 2, 4
P = 0x10000          # an aligned address that nothing reads


@pytest.fixture(scope="module")
def b():
    import os
    from paper_2410_06270_amd import _binding
    if not os.path.exists(_binding.lib_path()):
        from paper_2410_06270_amd import build
        build.build()
    _binding.load()
    return _binding


def cache(b, **kw):
    c = dict(n_pages=10, page=16, Hkv=2, D=64, dtype=0, k=P, v=P, page_stride=None, k_bytes=None, v_bytes=None,
             k_scale=None, v_scale=None)
    c.update(kw)
    per = c["page"] * c["Hkv"] * c["D"] * (1 if c["dtype"] else 2)
    if c["page_stride"] is None:
        c["page_stride"] = per
    full = (c["n_pages"] - 1) * c["page_stride"] + per
    for x in ("k_bytes", "v_bytes"):
        if c[x] is None:
            c[x] = full
        elif c[x] < 0:
            c[x] = full + c[x]
    return b._KVCache(*[c[n] for n, _ in b._KVCache._fields_])


def batch(b, **kw):
    c = dict(S=3, T=7, max_pages=4, max_len=0, q_start=P, kv_len=P, page_table=P)
    c.update(kw)
    return b._KVBatch(*[c[n] for n, _ in b._KVBatch._fields_])


def attention(b, **kw):
    c = dict(Hq=4, scale=0.125, softcap=0.0, window=0, slopes=None, prefix=None)
    c.update(kw)
    return b._Attention(*[c[n] for n, _ in b._Attention._fields_])


def prep(b, **kw):
    c = dict(q_norm=None, k_norm=None, norm_row=0, eps=1e-5, rot=0, rope_pairs=0, rope=None, n_pos=0)
    c.update(kw)
    return b._QKPrep(*[c[n] for n, _ in b._QKPrep._fields_])


BAD_CACHES = [
    (dict(page=8), EINVAL), (dict(page=48), EINVAL), (dict(page=512), EINVAL), (dict(Hkv=0), EINVAL),
    (dict(Hkv=257), EINVAL), (dict(D=96), EUNSUPPORTED), (dict(D=256), EUNSUPPORTED), (dict(D=100), EINVAL),
    (dict(D=0), EINVAL), (dict(dtype=2), EINVAL), (dict(n_pages=0), EINVAL), (dict(k=None), EINVAL),
    (dict(v=None), EINVAL), (dict(k=P + 8), EINVAL), (dict(v=P + 2), EINVAL),
    (dict(page_stride=4096 - 16), EINVAL), (dict(page_stride=4096 + 8), EINVAL), (dict(k_bytes=-1), ENOSPACE),
    (dict(v_bytes=-1), ENOSPACE), (dict(page_stride=(1 << 62)), ENOSPACE),
    (dict(dtype=1), EINVAL), (dict(dtype=1, k_scale=P), EINVAL), (dict(k_scale=P, v_scale=P), EINVAL),
]
BAD_BATCHES = [
    (dict(S=0), EINVAL), (dict(S=65537), EUNSUPPORTED), (dict(max_pages=0), EINVAL), (dict(max_len=-1), EINVAL),
    (dict(kv_len=None), EINVAL), (dict(page_table=None), EINVAL),
]
BAD_RAGGED = BAD_BATCHES + [(dict(T=0), EINVAL), (dict(T=65537), EUNSUPPORTED), (dict(q_start=None), EINVAL)]
BAD_ATTENTION = [
    (dict(Hq=0), EINVAL), (dict(Hq=5), EINVAL), (dict(Hq=258), EINVAL), (dict(scale=math.inf), EINVAL),
    (dict(scale=math.nan), EINVAL), (dict(softcap=-1.0), EINVAL), (dict(softcap=math.nan), EINVAL),
    (dict(softcap=math.inf), EINVAL), (dict(window=-1), EINVAL),
]


def need(b, ragged, Hq=4, Hkv=2, D=64):
    n = ctypes.c_size_t()
    assert b.load().mc_attn_workspace(7 if ragged else 3, Hq, Hkv, D, ctypes.byref(n)) == 0
    return n.value


def call(b, which, c=None, bt=None, a=None, q=P, qs=256, o=P, os=256, ws=P, ws_bytes=None):
    ragged = which == "prefill"
    c = c if c is not None else cache(b)
    bt = bt if bt is not None else batch(b)
    a = a if a is not None else attention(b)
    if ws_bytes is None:
        ws_bytes = need(b, ragged)
    f = getattr(b.load(), "mc_attn_" + which)
    ref = lambda t: None if t == "null" else ctypes.byref(t)  # noqa: E731
    return f(q, qs, ref(bt), ref(c), ref(a), o, os, None, ws, ws_bytes, None)


@pytest.mark.parametrize("which", ["decode", "prefill"])
def test_attention_refusals(b, which):
    for kw, want in BAD_CACHES:
        assert call(b, which, c=cache(b, **kw)) == want, kw
        assert b.load().mc_last_error()
    for kw, want in (BAD_RAGGED if which == "prefill" else BAD_BATCHES):
        assert call(b, which, bt=batch(b, **kw)) == want, kw
    for kw, want in BAD_ATTENTION:
        assert call(b, which, a=attention(b, **kw)) == want, kw
    for kw, want in [(dict(c="null"), EINVAL), (dict(bt="null"), EINVAL), (dict(a="null"), EINVAL),
                     (dict(q=None), EINVAL), (dict(o=None), EINVAL), (dict(q=P + 8), EINVAL), (dict(o=P + 4), EINVAL),
                     (dict(qs=248), EINVAL), (dict(qs=260), EINVAL), (dict(os=255), EINVAL), (dict(ws=None), EINVAL),
                     (dict(ws=P + 4), EINVAL), (dict(ws_bytes=need(b, which == "prefill") - 1), ENOSPACE),
                     (dict(ws_bytes=0), ENOSPACE)]:
        assert call(b, which, **kw) == want, kw


def append(b, c=None, bt=None, p=None, Hq=4, q=P, qs=512, k=P, ks=512, v=P, vs=512, out=P, os=256):
    c = c if c is not None else cache(b)
    bt = bt if bt is not None else batch(b)
    ref = lambda t: None if t is None or t == "null" else ctypes.byref(t)  # noqa: E731
    return b.load().mc_kv_append(q, qs, k, ks, v, vs, Hq, ref(p), ref(bt), ref(c), out, os, None)


def test_append_refusals(b):
    for kw, want in BAD_CACHES:
        assert append(b, c=cache(b, **kw)) == want, kw
    for kw, want in BAD_RAGGED:
        assert append(b, bt=batch(b, **kw)) == want, kw
    for kw, want in [(dict(Hq=0), EINVAL), (dict(Hq=257), EINVAL), (dict(q=None), EINVAL), (dict(out=None), EINVAL),
                     (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(q=P + 8), EINVAL), (dict(k=P + 8), EINVAL),
                     (dict(v=P + 8), EINVAL), (dict(out=P + 8), EINVAL), (dict(qs=248), EINVAL), (dict(ks=120), EINVAL),
                     (dict(vs=121), EINVAL), (dict(os=252), EINVAL), (dict(out=P, os=512 + 8), EINVAL)]:
        assert append(b, **kw) == want, kw
    for kw in (dict(q_norm=P), dict(k_norm=P), dict(q_norm=P + 8, k_norm=P), dict(q_norm=P, k_norm=P + 2),
               dict(eps=-1.0), dict(eps=math.nan), dict(rot=8, rope=P, n_pos=5), dict(rot=80, rope=P, n_pos=5),
               dict(rot=-16, rope=P, n_pos=5), dict(rot=32, n_pos=5), dict(rot=32, rope=P, n_pos=0),
               dict(rot=32, rope=P + 8, n_pos=5)):
        assert append(b, p=prep(b, **kw)) == EINVAL, kw


def importance(b, c=None, bt=None, a=None, q=P, qs=256, lse=P, x=P, d=64, rho=0.02, mask=P, ws=P, ws_bytes=None):
    c = c if c is not None else cache(b)
    bt = bt if bt is not None else batch(b, S=1, T=50)
    a = a if a is not None else attention(b)
    if ws_bytes is None:
        n = ctypes.c_size_t()
        assert b.load().mc_attn_importance_workspace(4, 50, ctypes.byref(n)) == 0
        ws_bytes = n.value
    ref = lambda t: None if t == "null" else ctypes.byref(t)  # noqa: E731
    return b.load().mc_attn_importance(q, qs, lse, ref(bt), ref(c), ref(a), x, d, ctypes.c_float(rho), None, mask, ws,
                                       ws_bytes, None)


def test_importance_refusals(b):
    for kw, want in BAD_CACHES:
        assert importance(b, c=cache(b, **kw)) == want, kw
    for kw, want in BAD_ATTENTION + [(dict(prefix=P), EUNSUPPORTED)]:
        assert importance(b, a=attention(b, **kw)) == want, kw
    for kw, want in [(dict(S=2, T=50), EINVAL), (dict(S=1, T=0), EINVAL), (dict(S=1, T=65537, max_pages=5000), EUNSUPPORTED),
                     (dict(S=1, T=65, max_pages=4), EINVAL), (dict(S=1, T=50, page_table=None), EINVAL)]:
        assert importance(b, bt=batch(b, **kw)) == want, kw
    for kw, want in [(dict(c="null"), EINVAL), (dict(bt="null"), EINVAL), (dict(a="null"), EINVAL),
                     (dict(q=None), EINVAL), (dict(qs=240), EINVAL), (dict(lse=None), EINVAL), (dict(x=None), EINVAL),
                     (dict(d=0), EINVAL), (dict(rho=-0.1), EINVAL), (dict(rho=1.1), EINVAL), (dict(rho=math.nan), EINVAL),
                     (dict(mask=None), EINVAL), (dict(ws=None), EINVAL), (dict(ws=P + 8), EINVAL),
                     (dict(ws_bytes=0), ENOSPACE)]:
        assert importance(b, **kw) == want, kw


def test_sizes_beyond_a_launch_or_a_position(b):
    """Tables of more than 2^30 positions and launches of 2^32 threads are refused; one
    less is not (it gets as far as the workspace, which is too small)."""
    for n, want in [((1 << 26) + 1, EUNSUPPORTED), ((1 << 31) - 1, EUNSUPPORTED), (1 << 26, ENOSPACE)]:
        for which in ("decode", "prefill"):
            assert call(b, which, bt=batch(b, max_pages=n), ws_bytes=0) == want, (which, n)
        assert importance(b, bt=batch(b, S=1, T=50, max_pages=n), ws_bytes=0) == want, n
    assert append(b, bt=batch(b, max_pages=(1 << 26) + 1)) == EUNSUPPORTED
    assert call(b, "decode", c=cache(b, page=256), bt=batch(b, max_pages=(1 << 22) + 1)) == EUNSUPPORTED
    c, a = cache(b, Hkv=256), attention(b, Hq=256)
    for which, S, T, want in [("decode", 65536, 0, EUNSUPPORTED), ("decode", 65535, 0, ENOSPACE),
                              ("prefill", 65536, 1, EUNSUPPORTED), ("prefill", 65408, 16384, EUNSUPPORTED),
                              ("prefill", 65407, 16384, ENOSPACE)]:
        assert call(b, which, c=c, a=a, bt=batch(b, S=S, T=T), qs=16384, os=16384, ws_bytes=0) == want, (which, S, T)


def test_importance_row_stride(b):
    for qs, want in [((1 << 24) + 8, EUNSUPPORTED), (1 << 24, ENOSPACE)]:
        assert importance(b, qs=qs, ws_bytes=0) == want, qs


def test_size_queries(b):
    lib, n = b.load(), ctypes.c_size_t()
    assert lib.mc_kv_page_bytes(16, 8, 128, 0, ctypes.byref(n)) == 0 and n.value == 16 * 8 * 128 * 2
    assert lib.mc_kv_page_bytes(256, 3, 64, 1, ctypes.byref(n)) == 0 and n.value == 256 * 3 * 64
    assert lib.mc_kv_page_bytes(16, 8, 128, 0, None) == EINVAL
    assert lib.mc_kv_page_bytes(20, 8, 128, 0, ctypes.byref(n)) == EINVAL
    for args, want in [((0, 4, 2, 64), EINVAL), ((1, 0, 1, 64), EINVAL), ((1, 3, 2, 64), EINVAL),
                       ((1, 4, 2, 80), EUNSUPPORTED), ((65537, 4, 2, 64), EUNSUPPORTED)]:
        assert lib.mc_attn_workspace(*args, ctypes.byref(n)) == want, args
    assert lib.mc_attn_workspace(1, 4, 2, 64, None) == EINVAL
    # a workspace serves every smaller batch
    last = 0
    for T in (1, 2, 3, 17, 64, 100, 256, 1000, 65536):
        assert lib.mc_attn_workspace(T, 32, 8, 128, ctypes.byref(n)) == 0
        assert n.value >= last
        last = n.value
    for args, want in [((0, 5), EINVAL), ((257, 5), EINVAL), ((4, 0), EINVAL), ((4, 65537), EUNSUPPORTED)]:
        assert lib.mc_attn_importance_workspace(*args, ctypes.byref(n)) == want, args


@pytest.mark.parametrize("U", [8, 16])
def test_oracle_layout(U):
    """Whole-row offsets agree with the header's formula, and fill a cache exactly."""
    page, Hkv, D = 32, 3, 64
    pages = torch.tensor([4, 0, 2, 1, 3])
    for w in "kv":
        seen = []
        for h in range(Hkv):
            rows = oa._offsets(w, pages, torch.arange(5 * page), h, page, Hkv, D, U)
            seen.append(rows.reshape(-1))
            for pos in (0, 7, 8, 15, 16, 31, 32, 100, 159):
                for i in (0, 1, 15, 16, 63):
                    assert int(rows[pos, i]) == oa.offset(w, int(pages[pos // page]), h, pos % page, i, page, Hkv, D, U)
        seen = torch.sort(torch.cat(seen)).values
        assert torch.equal(seen, torch.arange(5 * page * Hkv * D))


def test_oracle_attention_by_hand():
    """Two keys at scores 0 and ln 3, a window that hides the first, a row of nothing."""
    D = 64
    q = torch.zeros((1, D), dtype=torch.float64)
    q[0, 0] = 1.0
    k = torch.zeros((2, D), dtype=torch.float64)
    k[1, 0] = math.log(3.0)
    v = torch.arange(2 * D, dtype=torch.float64).view(2, D)
    o, lse, tol, _ = oa.attend(q, k, v, [1], scale=1.0)
    assert abs(float(lse) - math.log(4.0)) < 1e-14
    assert torch.allclose(o[0], 0.25 * v[0] + 0.75 * v[1], atol=1e-12) and bool((tol > 0).all())
    o, lse, _, _ = oa.attend(q, k, v, [1], scale=1.0, window=1)
    assert torch.equal(o[0], v[1]) and float(lse) == math.log(3.0)
    o, lse, _, _ = oa.attend(q, k, v, [-1], scale=1.0, prefix=2)
    assert bool((o == 0).all()) and float(lse) == -math.inf
    o, lse, _, _ = oa.attend(q, k, v, [0], scale=1.0, prefix=2)
    assert abs(float(lse) - math.log(4.0)) < 1e-14


def test_binding_refuses(b):
    """The binding's own checks of types and shapes."""
    with pytest.raises(AssertionError):
        b.kv_page_bytes(16, 2, 64, torch.float16)
    with pytest.raises(b.MCError):
        b.kv_page_bytes(24, 2, 64)
    t = torch.zeros((2, 4), dtype=torch.int32)
    with pytest.raises(AssertionError):
        b.KVBatch(torch.zeros(2, dtype=torch.int32), t)            # not on the GPU
    with pytest.raises(AssertionError):
        b.QKPrep(rope=torch.zeros((4, 16)))
    with pytest.raises(AssertionError):
        b.Attention(4, 0.1, slopes=torch.zeros(3))
