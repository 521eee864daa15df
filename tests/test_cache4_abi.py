"""Tables, the 4-bit cache and attention over selected pages: refusals, sizes and the oracle's own
rules, without a GPU."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

import test_attention_abi as t  # noqa: E402
from oracle import cache4 as o4  # noqa: E402

EINVAL, ENOSPACE, EUNSUPPORTED = 1, 2, 4
P = t.P
b = t.b              # the fixture that builds and loads the binding


def size(fn, *args):
    n = ctypes.c_size_t()
    return fn(*args, ctypes.byref(n)), n.value


def cache4(m, **kw):
    d = dict(n_pages=10, page=16, Hkv=2, D=64, dtype=4, k=P, v=P, k_scale=None, v_scale=None)
    d.update(kw)
    per = o4.page_bytes(d["page"], d["Hkv"], d["D"])
    d.setdefault("page_stride", per)
    full = (d["n_pages"] - 1) * d["page_stride"] + per
    d.setdefault("k_bytes", full)
    d.setdefault("v_bytes", full)
    return m._KVCache(*[d[n] for n, _ in m._KVCache._fields_])


def pool(m, **kw):
    d = dict(n_pages=8, page=16, free_list=P, n_free=P, n_free_out=P)
    d.update(kw)
    return m._KVPool(*[d[n] for n, _ in m._KVPool._fields_])


def tables(m, **kw):
    d = dict(S=3, T=7, max_pages=4, q_start=P, kv_len=P, page_table=P, positions=P, slots=P)
    d.update(kw)
    return m._KVTables(*[d[n] for n, _ in m._KVTables._fields_])


def summary(m, **kw):
    d = dict(bounds=P, scale=P, bounds_bytes=1 << 20, scale_bytes=1 << 20)
    d.update(kw)
    return m._KVSummary(*[d[n] for n, _ in m._KVSummary._fields_])


@pytest.mark.parametrize("page,Hkv,D", [(16, 1, 64), (64, 8, 128), (256, 256, 128), (32, 5, 64)])
def test_page_bytes(b, page, Hkv, D):
    assert size(b.load().mc_kv_page_bytes, page, Hkv, D, 4) == (0, o4.page_bytes(page, Hkv, D))
    assert size(b.load().mc_kv_page_bytes, page, Hkv, D, 3)[0] == EINVAL
    assert o4.page_bytes(page, Hkv, D) % 16 == 0


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("page,Hkv,D", [(16, 3, 64), (32, 2, 128)])
def test_layout_is_a_bijection(which, page, Hkv, D):
    """Every half of a code byte, and of the scale bytes each at most once, has one owner."""
    codes = {o4.code_place(which, h, x, i, page, D) for h in range(Hkv) for x in range(page) for i in range(D)}
    assert len(codes) == Hkv * page * D and max(c[0] for c in codes) == Hkv * page * D // 2 - 1
    step, width = (32, 1) if which == "k" else (64, 2)
    sc = [o4.scale_place(which, h, x, i, page, Hkv, D) for h in range(Hkv) for x in range(page)
          for i in range(0, D, step)]
    taken = {s + w for s in sc for w in range(width)}
    assert len(taken) == width * len(sc) and min(taken) == Hkv * page * D // 2
    assert max(taken) == o4.page_bytes(page, Hkv, D) - 1


def test_levels_and_borders():
    borders = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    even = [0, 2, 2, 4, 4, 6, 6]
    for x, e in zip(borders, even):
        got = o4.nearest(torch.tensor([x, math.nextafter(x, 0), math.nextafter(x, 9), -x], dtype=torch.float64))
        i = borders.index(x)
        assert got.tolist() == [e, i, i + 1, e + 8]
    assert o4.nearest(torch.tensor([100.0, 7.0, 6.0], dtype=torch.float64)).tolist() == [7, 7, 7]


@pytest.mark.parametrize("m,byte", [(7.0, 127), (math.nextafter(7.0, 8), 128), (3.5, 126), (2.0 ** -100, 25),
                                    (math.nextafter(2.0 ** -100, 0), 0), (7 * 2.0 ** 125, 252), (math.inf, 255),
                                    (math.nan, 255)])
def test_key_scale(m, byte):
    y = torch.zeros(64, dtype=torch.float64)
    y[5] = -m
    assert o4.quantize_keys(y)[1].tolist() == [byte, 0]


def test_every_value_is_a_bf16_number():
    g = torch.Generator().manual_seed(0)
    v = (torch.randn((50, 128), generator=g) * torch.exp(3 * torch.randn((50, 1), generator=g))).to(torch.bfloat16)
    x = o4.values("v", *o4.quantize_values(v))
    assert torch.equal(x, x.to(torch.bfloat16).double())
    # a level is off by at most half of the widest step between levels, 1/3 of 6, and by the scale's rounding
    assert float(((x - v.double()).abs() / v.double().abs().amax(1, keepdim=True)).max()) <= 1 / 6 + 2.0 ** -6


@pytest.mark.parametrize("kw,status", [
    (dict(k_scale=P, v_scale=P), EINVAL), (dict(k_scale=P), EINVAL), (dict(page_stride=512), EINVAL),
    (dict(page_stride=1096), EINVAL), (dict(k_bytes=10 * 1088 - 1), ENOSPACE), (dict(dtype=3), EINVAL),
    (dict(D=96), EUNSUPPORTED)])
def test_cache_refusals(b, kw, status):
    lib = b.load()
    bt, at = t.batch(b), t.attention(b)
    n = 1 << 30
    cc = cache4(b, **kw)
    assert lib.mc_attn_decode(P, 512, ctypes.byref(bt), ctypes.byref(cc), ctypes.byref(at), P, 512, None, P, n,
                              None) == status
    assert lib.mc_kv_read(ctypes.byref(bt), ctypes.byref(cc), P, 512, P, 512, None) == status


@pytest.mark.parametrize("batch,k,ks,v,vs,status", [
    (dict(), None, 0, None, 0, EINVAL), (dict(), P + 2, 128, None, 0, EINVAL), (dict(), P, 120, None, 0, EINVAL),
    (dict(), P, 132, None, 0, EINVAL), (dict(q_start=None), P, 128, P, 128, EINVAL),
    (dict(T=70000), P, 128, P, 128, EUNSUPPORTED), (dict(T=0), P, 128, P, 128, EINVAL)])
def test_read_refusals(b, batch, k, ks, v, vs, status):
    bt, cc = t.batch(b, **batch), cache4(b)
    assert b.load().mc_kv_read(ctypes.byref(bt), ctypes.byref(cc), k, ks, v, vs, None) == status


@pytest.mark.parametrize("p,tb,want,past,ws,n,status", [
    (dict(page=24), {}, P, P, P, 1 << 20, EINVAL), (dict(page=8), {}, P, P, P, 1 << 20, EINVAL),
    (dict(n_pages=0), {}, P, P, P, 1 << 20, EINVAL), (dict(free_list=None), {}, P, P, P, 1 << 20, EINVAL),
    (dict(n_pages=(1 << 30) + 1), {}, P, P, P, 1 << 20, EUNSUPPORTED),
    (dict(n_free=None), {}, P, P, P, 1 << 20, EINVAL), (dict(n_free_out=None), {}, P, P, P, 1 << 20, EINVAL),
    ({}, dict(S=0), P, P, P, 1 << 20, EINVAL), ({}, dict(S=70000), P, P, P, 1 << 20, EUNSUPPORTED),
    ({}, dict(max_pages=0), P, P, P, 1 << 20, EINVAL),
    ({}, dict(max_pages=(1 << 26) + 1), P, P, P, 1 << 20, EUNSUPPORTED),
    ({}, dict(kv_len=None), P, P, P, 1 << 20, EINVAL), ({}, dict(page_table=None), P, P, P, 1 << 20, EINVAL),
    ({}, {}, P, None, P, 1 << 20, EINVAL), ({}, {}, None, P, P, 1 << 20, EINVAL), ({}, {}, P, P, None, 1 << 20, EINVAL),
    ({}, {}, P, P, P + 2, 1 << 20, EINVAL), ({}, {}, P, P, P, 27, ENOSPACE)])
def test_tables_refusals(b, p, tb, want, past, ws, n, status):
    lib, po, ta = b.load(), pool(b, **p), tables(b, **tb)
    assert lib.mc_kv_reserve(want, past, ctypes.byref(po), ctypes.byref(ta), ws, n, None) == status
    assert lib.mc_kv_release(want, past, ctypes.byref(po), ctypes.byref(ta), ws, n, None) == status


@pytest.mark.parametrize("tb,status", [(dict(T=0), EINVAL), (dict(T=70000), EUNSUPPORTED), (dict(q_start=None), EINVAL),
                                       (dict(slots=P + 4), EINVAL)])
def test_reserve_refusals(b, tb, status):
    po, ta = pool(b), tables(b, **tb)
    assert b.load().mc_kv_reserve(P, P, ctypes.byref(po), ctypes.byref(ta), P, 1 << 20, None) == status
    assert b.load().mc_kv_reserve(P, P, None, ctypes.byref(ta), P, 1 << 20, None) == EINVAL


def test_workspaces(b):
    lib = b.load()
    assert size(lib.mc_kv_tables_workspace, 3) == (0, 28)
    assert size(lib.mc_kv_tables_workspace, 0)[0] == EINVAL
    assert size(lib.mc_kv_tables_workspace, 65537)[0] == EUNSUPPORTED
    assert size(lib.mc_attn_select_workspace, 4, 2, 100) == (0, 4 * 2 * 100 * 4)
    # long prompts: in parts of 256 MB, or of one row
    assert size(lib.mc_attn_select_workspace, 65536, 8, 8192) == (0, 256 << 20)
    assert size(lib.mc_attn_select_workspace, 5, 256, 1 << 26) == (0, 256 << 28)
    for bad in ((0, 2, 3), (1, 0, 3), (1, 257, 3), (1, 2, 0)):
        assert size(lib.mc_attn_select_workspace, *bad)[0] == EINVAL
    assert size(lib.mc_attn_select_workspace, 65537, 1, 1)[0] == EUNSUPPORTED
    assert size(lib.mc_attn_select_workspace, 1, 1, (1 << 26) + 1)[0] == EUNSUPPORTED


@pytest.mark.parametrize("kw,status", [
    (dict(sm=dict(bounds=None)), EINVAL), (dict(sm=dict(scale=None)), EINVAL), (dict(sm=dict(bounds=P + 8)), EINVAL),
    (dict(sm=dict(bounds_bytes=10 * 2 * 128 - 1)), ENOSPACE), (dict(sm=dict(scale_bytes=79)), ENOSPACE),
    (dict(bt=dict(kv_len=None)), EINVAL), (dict(bt=dict(page_table=None)), EINVAL), (dict(bt=dict(S=0)), EINVAL)])
def test_summary_refusals(b, kw, status):
    bt, cc, sm = t.batch(b, **kw.get("bt", {})), cache4(b), summary(b, **kw.get("sm", {}))
    at = t.attention(b)
    lib = b.load()
    assert lib.mc_kv_summarize(ctypes.byref(bt), ctypes.byref(cc), ctypes.byref(sm), None) == status
    assert lib.mc_attn_select(P, 256, ctypes.byref(bt), ctypes.byref(cc), ctypes.byref(sm), ctypes.byref(at), 4, 1, 1, P,
                              P, P, 1 << 20, None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), EINVAL), (dict(n=4097), EUNSUPPORTED), (dict(first=-1), EINVAL), (dict(last=0), EINVAL),
    (dict(first=4), EINVAL), (dict(first=2, last=3), EINVAL), (dict(first=2 ** 31 - 1), EINVAL), (dict(sel=None), EINVAL),
    (dict(count=None), EINVAL), (dict(q=None), EINVAL), (dict(stride=248), EINVAL), (dict(at=dict(prefix=P)), EUNSUPPORTED),
    (dict(at=dict(slopes=P)), EUNSUPPORTED), (dict(at=dict(Hq=5)), EINVAL), (dict(ws=None), EINVAL),
    (dict(ws_n=7 * 2 * 4 * 4 - 1), ENOSPACE), (dict(bt=dict(T=65536, max_pages=1 << 20)), EUNSUPPORTED)])
def test_select_refusals(b, kw, status):
    bt, cc, sm = t.batch(b, **kw.get("bt", {})), cache4(b), summary(b)
    at = t.attention(b, **kw.get("at", {}))
    assert b.load().mc_attn_select(kw.get("q", P), kw.get("stride", 256), ctypes.byref(bt), ctypes.byref(cc),
                                   ctypes.byref(sm), ctypes.byref(at), kw.get("n", 4), kw.get("first", 1),
                                   kw.get("last", 1), kw.get("sel", P), kw.get("count", P), kw.get("ws", P),
                                   kw.get("ws_n", 1 << 20), None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), EINVAL), (dict(n=4097), EUNSUPPORTED), (dict(sel=None), EINVAL), (dict(count=None), EINVAL),
    (dict(q=None), EINVAL), (dict(o=None), EINVAL), (dict(at=dict(prefix=P)), EUNSUPPORTED), (dict(ws=None), EINVAL),
    (dict(ws=P + 8), EINVAL), (dict(ws_n=16), ENOSPACE), (dict(bt=dict(T=0)), EINVAL),
    (dict(bt=dict(T=65537)), EUNSUPPORTED)])
def test_sparse_refusals(b, kw, status):
    bt, cc, at = t.batch(b, **kw.get("bt", {})), cache4(b), t.attention(b, **kw.get("at", {}))
    assert b.load().mc_attn_sparse(kw.get("q", P), 256, ctypes.byref(bt), ctypes.byref(cc), ctypes.byref(at),
                                   kw.get("sel", P), kw.get("count", P), kw.get("n", 4), kw.get("o", P), 256, None,
                                   kw.get("ws", P), kw.get("ws_n", 1 << 30), None) == status


def test_reserve_rules():
    """By hand: page 16, five free pages 10 .. 14 (14 on top), rows of up to 3 pages."""
    table = torch.full((5, 3), -1, dtype=torch.int32)
    free = [10, 11, 12, 13, 14]
    # 0: 1 -> 2 pages;  1: too long for its row;  2: needs three;  3: needs two more than there are;  4: none
    got = o4.reserve([16, 20, 40, 33, 3], [10, 40, 0, 0, 1], free, 5, table, 16, 100)
    assert got[0] == [0, 16, 16, 56, 56, 59] and got[1] == [26, 40, 40, 0, 4] and got[4] == 1
    assert table.tolist() == [[-1, 14, -1], [-1] * 3, [13, 12, 11], [-1] * 3, [-1] * 3]
    assert got[2][:17] == list(range(10, 26)) + [0] and got[3][6] == 14 * 16 and got[3][16] == 13 * 16
    # rows run out: 2 would need the 56th row
    got = o4.reserve([16, 0, 40, 1, 1], [10, 0, 0, 15, 1], free, 5, table, 16, 55)
    assert got[0] == [0, 16, 16, 16, 16, 16] and got[4] == 4 and got[2][16] == -1 and len(got[2]) == 55


def test_release_rules():
    free = [3, 0, 0, 0]
    table = torch.tensor([[7, 8], [1, 2], [5, 6]], dtype=torch.int32)
    assert o4.release([1, 0, 1], [17, 20, 16], free, 1, table, 16) == ([0, 20, 0], 4)
    assert free == [3, 7, 8, 5]
    assert o4.release([1, 1, 1], [32, 32, 32], free, 3, table, 16) == ([0, 0, 0], 4) and free == [3, 7, 8, 7]


def test_binding_asserts(b):
    """Tensors that are not on a GPU, of another type or shape."""
    i = torch.zeros(4, dtype=torch.int32)
    for args in ((16, i, i), (16, i.long(), i[:1]), (16, i, i[:1].float())):
        with pytest.raises(AssertionError):
            b.KVPool(*args)
    with pytest.raises(AssertionError):
        b.KVCache(2, 16, 1, 64, dtype=torch.float4_e2m1fn_x2, k=torch.zeros((2, 544), dtype=torch.uint8),
                  v=torch.zeros((2, 544), dtype=torch.uint8))        # not on the GPU
    with pytest.raises(AssertionError):
        b.kv_page_bytes(16, 1, 64, torch.float16)
    assert b.kv_page_bytes(16, 1, 64, torch.float4_e2m1fn_x2) == 544


def test_many_rows_refused(b):
    """Launches of 2^24 workgroups and more."""
    lib = b.load()
    bt, cc, sm = t.batch(b, S=65536, T=65536), cache4(b, Hkv=256), summary(b, bounds_bytes=1 << 30, scale_bytes=1 << 30)
    at = t.attention(b, Hq=256)
    r = ctypes.byref
    assert lib.mc_kv_summarize(r(bt), r(cc), r(sm), None) == EUNSUPPORTED
    assert lib.mc_attn_select(P, 1 << 14, r(bt), r(cc), r(sm), r(at), 4, 1, 1, P, P, P, 1 << 40, None) == EUNSUPPORTED
    assert lib.mc_attn_sparse(P, 1 << 14, r(bt), r(cc), r(at), P, P, 4, P, 1 << 14, None, P, 1 << 40, None) == EUNSUPPORTED
