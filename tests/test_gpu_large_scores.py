"""Scores far beyond what a softmax tells apart, yet finite in 32 bits (mla_cache_attend): the
keys of the largest score are answered, not NaN."""
import numpy as np
import pytest

import mx4_reference as R
from test_gpu_cache import _bf16_dev, _dev, _host, own, random_cache, run_attend, table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,n", [(4, 70), (24, 30), (64, 200)])
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 14, 2.0 ** 17, 2.0 ** 20, 2.0 ** 40])
def test_large_scores(heads, n, size):
    """Queries and latents of this size: one key of a request scores far above the others,
    which lie on the other side of 0, so a row's answer is that key's latent."""
    import torch
    rng = np.random.default_rng(heads + n)
    sign = np.where(rng.random(512) < 0.5, -1.0, 1.0)
    lat = -sign * rng.choice([0.5, 1.0, 1.5, 3.0, 6.0], (n, 512)) * size
    best = n // 2
    lat[best] = -lat[best]
    c, s = R.quantize(R.bf16(lat))
    per = -(-n // 64)
    raw = random_cache(rng, per, 64)
    codes = np.zeros((per * 64, 256), dtype=np.uint8)
    scales = np.full((per * 64, 16), 127, dtype=np.uint8)
    codes[:n], scales[:n] = R.pack(c), s
    raw[:, : 64 * 256], raw[:, 64 * 256: 64 * 272] = codes.reshape(per, -1), scales.reshape(per, -1)
    q = rng.standard_normal((1, 1, heads, 576))
    q[..., :512] = sign * (1 + rng.random((1, 1, heads, 512))) * size
    pages, count = table([own(n)], 64, np.arange(per))
    out, lse = run_attend(R.geom(heads), _bf16_dev(q), _dev(np.array([[n - 1]], dtype=np.int32)), _dev(pages), _dev(count), _dev(raw), 64)
    lse = lse.cpu().numpy()
    assert np.isfinite(lse).all()
    # one weight of all is not 0: its value is answered as it is
    assert np.array_equal(_host(out)[0, 0], np.broadcast_to(R.values(c, s)[best], (heads, 512)))
    x = _host(_bf16_dev(q))[0, 0]
    score = x[:, :512] @ R.values(c, s)[best] / np.sqrt(192.0)
    assert (np.abs(lse[0, 0] - score) <= 2.0 ** -14 * np.abs(score)).all()   # 576 products in 32-bit sums
