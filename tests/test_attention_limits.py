"""Scales and caps that the attention calls take: up to 2^126, on the host (no GPU)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from test_attention_abi import ENOSPACE, EUNSUPPORTED, attention, b, call, importance  # noqa: E402,F401

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
