"""GPU test of what the header says of rows whose softmax is no number (mla_moe_route): one NaN or +infinity makes every score of
the row NaN."""
import numpy as np
import pytest

from test_gpu_route import _route

pytestmark = pytest.mark.gpu


def rows(e, bad, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((50, e)).astype(np.float32)
    x[np.arange(50), rng.integers(0, e, 50)] = bad
    return x, rng


def by_logit(x, allowed):
    """allowed experts of a row from the largest logit down, NaN last, equal ones by index."""
    return sorted(allowed, key=lambda i: (np.isnan(x[i]), -x[i] if not np.isnan(x[i]) else 0.0, i))


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("e,groups", [(64, dict()), (64, dict(n_groups=8, top_groups=3)), (256, dict(n_groups=8, top_groups=4, group_best=2)), (600, dict())])
def test_softmax(e, groups, bad):
    x, rng = rows(e, bad, e)
    k, kept = 6, groups.get("top_groups", 1) * (e // groups.get("n_groups", 1))
    # no bias: the lowest groups, in them the order of the logits
    _, idx, w, fan, _ = _route(x, k, None, scoring="softmax", min_k=2, tau=0.1, **groups)
    assert np.array_equal(idx, [by_logit(r, range(kept))[:k] for r in x])
    assert np.isnan(w).all() and (fan == k).all()
    # a bias: every c is NaN, the lowest experts
    _, idx, w, fan, _ = _route(x, k, rng.standard_normal(e), scoring="softmax", min_k=2, tau=0.1, **groups)
    assert np.array_equal(idx, np.tile(np.arange(k), (50, 1)))
    assert np.isnan(w).all() and (fan == k).all()


@pytest.mark.parametrize("bias", [None, 0.0])
def test_sigmoid(bias):
    """Each score by itself: the NaN comes last, +infinity has score 1."""
    for bad in (np.nan, np.inf):
        x, _ = rows(64, bad, 5)
        _, idx, w, fan, _ = _route(x, 6, None if bias is None else np.zeros(64), scoring="sigmoid", renormalize=False)
        assert np.array_equal(idx, [by_logit(r, range(64))[:6] for r in x]) and np.isfinite(w).all()
