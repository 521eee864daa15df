"""The limit of mc_attn_select's launch is the one that the header states, for groups that divide the
16 columns of a product and others."""
import ctypes
import os
from math import ceil, floor  # noqa: F401 (the formulas below)

import pytest

torch = pytest.importorskip("torch")

import test_attention_abi as t  # noqa: E402
import test_cache4_abi as t4  # noqa: E402

EINVAL, EUNSUPPORTED = 1, 4
P = t.P
b = t.b              # the fixture that builds and loads the binding
LIMIT = "tiles*Hkv*(ceil(max_pages/64) + 1)"
RAGGED = "ceil(T/max(1, floor(16/g))) + S - 1"


def status(b, g, Hkv, S, T, max_pages, ragged):
    """What the call says to a missing workspace, which it looks at last: EINVAL, or that it is too large."""
    bt = t.batch(b, S=S, T=T, max_pages=max_pages, **({} if ragged else dict(q_start=None)))
    cc, sm, at = t4.cache4(b, Hkv=Hkv), t4.summary(b), t.attention(b, Hq=g * Hkv)
    r = ctypes.byref
    return b.load().mc_attn_select(P, 64 * g * Hkv, r(bt), r(cc), r(sm), r(at), 4, 1, 1, P, P, None, 0, None)


def test_header_states_it():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mc_moe.h")
    with open(path) as f:
        text = " ".join(line.strip().lstrip("*").strip() for line in f)
    assert LIMIT in text and RAGGED in text


@pytest.mark.parametrize("Hkv", [1, 3])
@pytest.mark.parametrize("S", [1, 7])
@pytest.mark.parametrize("g", [1, 2, 3, 4, 5, 6, 7, 8, 9, 15, 16, 17, 40])
def test_ragged(b, g, S, Hkv):
    max_pages = 64 * 8000 - 5
    hit = {EINVAL: 0, EUNSUPPORTED: 0}
    R = max(1, 16 // g)
    most = (2 ** 24 - 1) // (Hkv * 8001)                  # tiles
    for T in (1, R * (most - S), R * (most - S + 1), R * (most - S + 1) + 1, R * (most - S + 3)):
        tiles = eval(RAGGED)
        want = EUNSUPPORTED if eval(LIMIT) >= 2 ** 24 else EINVAL
        assert status(b, g, Hkv, S, T, max_pages, True) == want, (T, tiles)
        hit[want] += 1
    assert hit == {EINVAL: 3, EUNSUPPORTED: 2}


@pytest.mark.parametrize("g", [1, 5, 9, 16])
def test_one_row_a_sequence(b, g):
    Hkv, max_pages = 2, 64 * 8000
    most = (2 ** 24 - 1) // (Hkv * 8001)
    for S, T in ((most, 1), (most + 1, 1), (most, 65536)):
        tiles = S
        want = EUNSUPPORTED if eval(LIMIT) >= 2 ** 24 else EINVAL
        assert status(b, g, Hkv, S, T, max_pages, False) == want == (EINVAL if S == most else EUNSUPPORTED)
