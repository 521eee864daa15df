"""What the score of a page bounds, by the oracle's rules (the kernels' bounds and selections are equal to them):
the products of the page's finite keys with the rounded query, up to the rounding of the scale."""
import pytest

torch = pytest.importorskip("torch")

from oracle import cache4 as o4  # noqa: E402

STEP = 2.0 ** -23


def score(q, k):
    """(score, rounded query as doubles) of one head's query q [D] for a page of keys k [n][D]."""
    lo, hi, s = o4.bounds(k)
    sq = q.abs().max() * o4._127TH
    q8 = (q / (sq if sq > 0 else torch.tensor(1.0))).round().clamp(-127, 127).long()
    whole = int((q8.clamp(min=0) * hi + q8.clamp(max=0) * lo).sum())
    return float(torch.tensor(float(whole)) * (sq * s)), q8.double() * float(sq)


def test_the_largest_key_may_pass_its_bound_by_a_rounding():
    """scale = max|k| fp32(1/127), two roundings of 2^-24: 127 of it may lie below max|k|, where the quotient's
    ceiling would be 128 and is cut."""
    short, cut = [], 0
    for m in torch.arange(128, 256).float() / 128:           # every bf16 mantissa
        for sign in (1.0, -1.0):
            lo, hi, s = o4.bounds(torch.tensor([[sign * float(m), 0.0]]))
            got = float(hi[0] if sign > 0 else -lo[0]) * float(s)
            short.append((float(m) - got) / float(m))
            cut += bool((m / s).ceil() > 127)
    assert 0 < max(short) <= STEP and cut > 0


@pytest.mark.parametrize("shift", [0, 40, -60])
def test_products_stay_below_the_score(shift):
    """A bound n s falls short of its key by 2^-23 max|k| at most (the clamp; 2^-24 where the quotient is rounded
    down to n), the score is rounded twice: 2^-22 of sum |q_i| max|k| in all, and as much again."""
    g = torch.Generator().manual_seed(shift + 100)
    for i in range(200):
        D, n = (64, 128)[i % 2], 1 + i % 16
        k = (torch.randn((n, D), generator=g) * 2.0 ** shift).to(torch.bfloat16).float()
        if i % 3 == 0:                                       # all keys at the ends of their range
            k = k.abs().amax() * torch.sign(k)
        q = torch.randn(D, generator=g).to(torch.bfloat16).float()
        got, qr = score(q, k)
        products = k.double() @ qr
        room = 2 * 2.0 ** -22 * float(qr.abs().sum()) * float(k.abs().max())
        assert float(products.max()) <= got + room


def test_keys_that_are_no_numbers_do_not_count():
    k = torch.tensor([[1.0, float("inf")], [float("nan"), -2.0]])
    lo, hi, s = o4.bounds(k)
    assert float(s) == float(torch.tensor(2.0) * o4._127TH)
    assert hi.tolist() == [64, -127] and lo.tolist() == [63, -127]
