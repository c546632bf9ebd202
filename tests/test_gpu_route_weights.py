"""GPU tests of the router's softmax weights (mla_moe_route) where the sum's errors weigh most, at the header's bound 2^-19, 32 steps of
2^-24, for up to 1024 experts.

A score takes its exponential, 2 steps, and the difference's own rounding put back, 1.  A term of the sum at a distance d from the
largest logit is off by 2.22 d + 2: the difference and its product with log2(e) are rounded to a step of d each, that constant is
off by 0.22, the exponential 2.  Weighted by e^-d, d is W((E - 1) / e) on average at most, where all others lie at one more than
that: 3.34 for 256 experts, 4.44 for 1024; the sum is off by 2.22 * 4.44 + 2 = 11.9.  Its terms are added up in 3 + 2 + 4
roundings (16 lanes of 16) or 3 + 2 + 6 (64 lanes).  The reciprocal takes 2, its product and the scale 1 each: 3 + 11.9 + 11 + 4 = 29.9."""
import numpy as np
import pytest

from test_gpu_route import check

pytestmark = pytest.mark.gpu

MEAN = {64: 2.31, 256: 3.34, 512: 3.88, 1024: 4.44}   # W((E - 1) / e)


def test_means():
    for e, m in MEAN.items():
        assert abs(m * np.exp(m) - (e - 1) / np.e) < 0.02 * e
        d = np.linspace(0.1, 12, 5000)
        share = (e - 1) * np.exp(-d)
        assert abs((d * share / (1 + share)).max() - m) < 0.01


@pytest.mark.parametrize("scale", [1.0, 2.5])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("e", list(MEAN))
def test_others_at_one_distance(e, bf16, scale):
    """All others equal, so that their errors are too; and in steps of a rounding around there, and logits of any size."""
    rng = np.random.default_rng(e)
    n = 3000
    d = MEAN[e] + 1 + rng.uniform(-1.5, 1.5, (n, 1))
    top = rng.uniform(-1, 1, (n, 1)) * 2.0 ** rng.integers(-8, 8, (n, 1))
    x = np.repeat(top - d, e, 1)
    x[n // 2:] += rng.uniform(-0.01, 0.01, (n - n // 2, e))
    x[np.arange(n), rng.integers(0, e, n)] = top[:, 0]
    check(x, 6, None, bf16=bf16, scoring="softmax", renormalize=False, min_k=6, scale=scale)
    check(x, 6, None, bf16=bf16, scoring="softmax", renormalize=True, min_k=6, scale=scale)
    check(x, 6, rng.standard_normal(e) * 0.3 / e, bf16=bf16, scoring="softmax", renormalize=False, min_k=6, scale=scale)
