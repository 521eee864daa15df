"""Selection and attention to selected pages without row starts: one row a sequence, whatever T the
batch was given, and nothing behind the last."""
import pytest

torch = pytest.importorskip("torch")

import test_gpu_attention as ta  # noqa: E402
import test_gpu_sparse as ts  # noqa: E402

pytestmark = pytest.mark.gpu

mc = ta.mc
BF16 = torch.bfloat16


@pytest.mark.parametrize("kind", [ts.BF16, ts.E4M3, ts.E2M1])
def test_rows_are_the_sequences(mc, kind):
    lens, Hq, Hkv, D, n_sel, more = [90, 1, 260, 0, 47], 4, 2, 64, 3, 4
    w = ts.world(mc, kind, lens, Hkv=Hkv, D=D, page=16, seed=3)
    sm = ts.summarize_all(mc, w, lens)
    S = len(lens)
    q = w.randn(S, Hq * D).to(BF16).cuda()
    kv_len, table = torch.tensor(lens, dtype=torch.int32, device="cuda"), w.table.cuda()
    attn = mc.Attention(Hq, D ** -0.5)
    ws = torch.zeros(max(mc.attn_select_workspace(16, Hkv, table.shape[1]), mc.attn_workspace(16, Hq, Hkv, D)),
                     dtype=torch.uint8, device="cuda")
    got = []
    for T in (None, 2, 9):
        batch = mc.KVBatch(kv_len, table, T=T)
        sel = torch.full((S + more, Hkv, n_sel), 77, dtype=torch.int32, device="cuda")
        count = torch.full((S + more, Hkv), 77, dtype=torch.int32, device="cuda")
        o = torch.full((S + more, Hq * D), 7.0, dtype=BF16, device="cuda")
        lse = torch.full((S + more, Hq), 7.0, device="cuda")
        print("rows", kind, T, flush=True)
        mc.attn_select(q, batch, w.cache, sm, attn, sel[:S], count[:S], ws)
        mc.attn_sparse(q, batch, w.cache, attn, sel[:S], count[:S], o[:S], ws, lse=lse[:S])
        torch.cuda.synchronize()
        assert bool((sel[S:] == 77).all()) and bool((count[S:] == 77).all())
        assert bool((o[S:] == 7.0).all()) and bool((lse[S:] == 7.0).all())
        got.append((sel.cpu(), count.cpu(), o.cpu(), lse.cpu()))
    assert got[0][1][:S].tolist() == [[3, 3], [1, 1], [3, 3], [0, 0], [3, 3]]
    for other in got[1:]:
        assert all(torch.equal(x, y) for x, y in zip(got[0], other))
