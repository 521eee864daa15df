"""Scales, caps and windows that the attention calls take, on the host (no GPU)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from test_attention_abi import EINVAL, ENOSPACE, EUNSUPPORTED, attention, b, call, importance  # noqa: E402,F401

MOST = 2.0 ** 126
ABOVE = MOST * (1 + 2.0 ** -23)


@pytest.mark.parametrize("kw,want", [
    (dict(softcap=MOST), ENOSPACE), (dict(softcap=ABOVE), EUNSUPPORTED), (dict(softcap=3.4e38), EUNSUPPORTED),
    (dict(scale=MOST), ENOSPACE), (dict(scale=-MOST), ENOSPACE), (dict(scale=ABOVE), EUNSUPPORTED),
    (dict(scale=-3.4e38), EUNSUPPORTED),
])
def test_scales_and_caps_beyond_the_log2_domain(b, kw, want):
    """What is accepted gets as far as the workspace, which is too small."""
    assert ctypes.c_float(ABOVE).value == ABOVE
    for which in ("decode", "prefill"):
        assert call(b, which, a=attention(b, **kw), ws_bytes=0) == want, which
    assert importance(b, a=attention(b, **kw), ws_bytes=0) == want


@pytest.mark.parametrize("window,want", [(0, 0), (4096, 4096), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1),
                                         (2 ** 32 + 5, 2 ** 31 - 1), (-1, -1), (-2 ** 32 + 5, -1)])
def test_windows_past_an_int(b, window, want):
    """Python's numbers do not wrap round: past the largest int they are that, below 0 refused."""
    assert b.Attention(4, 0.125, window=window).desc.window == want
    for which in ("decode", "prefill"):
        at = attention(b, window=b.Attention(4, 0.125, window=window).desc.window)
        assert call(b, which, a=at, ws_bytes=0) == (EINVAL if window < 0 else ENOSPACE)
