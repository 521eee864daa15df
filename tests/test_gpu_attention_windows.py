"""Importance under windows that hide nothing."""
import math

import pytest

torch = pytest.importorskip("torch")

from test_gpu_attention import BF16, mc  # noqa: E402,F401
from test_gpu_attention_block import Heads  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [333, 500])
def test_windows_of_everything_importance(mc, window):
    """A window as long as the sequence or longer: importance and its mask are those of no window."""
    L, Hq, Hkv, D, rho = 333, 4, 2, 64, 0.1
    outs = []
    for w in (0, window):
        h = Heads(mc, [L], Hq, Hkv, D, seed=3, window=w)
        gen = torch.Generator().manual_seed(4)
        qkv = torch.randn((L, (Hq + 2 * Hkv) * D), generator=gen).to(BF16).cuda()
        x = torch.randn((L, 64), generator=gen).to(BF16).cuda()
        q, o = (torch.empty((L, Hq * D), dtype=BF16, device="cuda") for _ in range(2))
        lse, imp = torch.empty((L, Hq), device="cuda"), torch.empty(L, device="cuda")
        mask, b = torch.empty(L, dtype=torch.uint8, device="cuda"), h.batch([L], [L])
        h.append(qkv, b, q)
        mc.attn_prefill(q, b, h.cache, h.attn, o, h.workspace(L), lse=lse)
        ws = torch.empty(mc.attn_importance_workspace(Hq, L), dtype=torch.uint8, device="cuda")
        mc.attn_importance(q, lse, b, h.cache, h.attn, x, rho, mask, ws, importance=imp)
        torch.cuda.synchronize()
        outs.append([t.cpu() for t in (lse, imp, mask)])
    (l0, i0, m0), (l1, i1, m1) = outs
    # lse: sums of up to 333 terms on either side; a probability moves by lse's difference, and
    # the sums of 4 heads' 333 rows and 64 values of x on either side are off by as many roundings
    far = float((l0 - l1).abs().max())
    assert far <= 2 * (L + 24) * 2.0 ** -24
    rel = 1.01 * (far + 2 * (L * Hq + 64 + 64) * 2.0 ** -24)
    assert bool(((i0.double() - i1).abs() <= rel * i0).all())
    n = int(math.floor(rho * L + 0.5))
    cut = float(torch.sort(i0, descending=True).values[n - 1])
    apart = (i0 - cut).abs() > 2 * rel * cut
    assert torch.equal(m0[apart], m1[apart]) and int(m0.sum()) == int(m1.sum()) == n
