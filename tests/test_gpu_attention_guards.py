"""What the cache and attention calls leave alone: memory around their outputs and cache
pages that no table names, whatever the device arrays hold."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_attention import BF16, mc  # noqa: E402,F401
from test_gpu_attention_block import i32  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_len", [1, 0])
@pytest.mark.parametrize("starts", [[0, 1, 2, 3], [0, 2, 1, 3], [-4, 1, 2, 3], [0, 1, 2, 900], [5, 5, 5, 5], [3, 2, 1, 0],
                                    [-2 ** 31, 0, 2 ** 31 - 1, 3], [2 ** 31 - 1] * 4])
def test_stray_starts_leave_the_rest(mc, starts, max_len):
    """Starts that are not ascending, negative or beyond the rows, with stray pages and
    lengths: outputs lie between guards, pages between others, and one is in no table."""
    Hq, Hkv, D, page, T, n_pages = 2, 1, 64, 16, 3, 6
    per = page * Hkv * D
    gen = torch.Generator().manual_seed(7)
    kbig, vbig = (torch.randn((n_pages + 4, 2 * per), generator=gen).to(BF16).cuda() for _ in range(2))
    cache = mc.KVCache(n_pages, page, Hkv, D, k=kbig[2:2 + n_pages, :per], v=vbig[2:2 + n_pages, :per])
    table = i32([[99, -5, 2 ** 31 - 1, -2 ** 31], [1, 5, 0, 3], [2, 2, 2, 2]])
    b = mc.KVBatch(i32([60, 50, 2 ** 31 - 1]), table, q_start=i32(starts), T=T, max_len=max_len)
    x = torch.randn((T, 4 * D), generator=gen).to(BF16).cuda()
    wide = 2 * Hq * D
    out = [torch.full((T + 8, wide), 7.0, dtype=BF16, device="cuda") for _ in range(2)]
    lse = torch.full((T + 8, Hq), 7.0, device="cuda")
    at = mc.Attention(Hq, D ** -0.5)
    ws = torch.empty(mc.attn_workspace(T, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    rows = slice(4, 4 + T)

    def guarded(t, mine):
        assert bool((t[:4] == 7.0).all()) and bool((t[4 + T:] == 7.0).all())
        assert mine is None or bool((t[:, mine:] == 7.0).all())

    was = [t.clone() for t in (kbig, vbig)]
    mc.attn_prefill(x[:, :2 * D], b, cache, at, out[0][rows, :Hq * D], ws, lse=lse[rows])
    torch.cuda.synchronize()
    guarded(out[0], Hq * D)
    guarded(lse, None)
    assert all(torch.equal(t, w) for t, w in zip((kbig, vbig), was))          # reads only
    mc.kv_append(x[:, :2 * D], x[:, 2 * D:3 * D], x[:, 3 * D:], None, b, cache, out[1][rows, :Hq * D])
    torch.cuda.synchronize()
    guarded(out[1], Hq * D)
    for t, w in zip((kbig, vbig), was):
        same = (t.view(torch.int16) == w.view(torch.int16)).view(n_pages + 4, 2, per).all(2).cpu()
        changed = torch.nonzero(~same).tolist()
        # pages 0, 1, 2, 3 and 5 are named; 4 and the layer beside are not
        assert all(half == 0 and p - 2 in (0, 1, 2, 3, 5) for p, half in changed), changed
    if starts == [0, 1, 2, 3]:            # (sequence 0 has no page; 1 is at token 49, 2 past its table)
        assert torch.equal(out[1][5, :Hq * D], x[1, :2 * D]) and bool((out[1][4] == 7.0).all())
