"""Several new tokens of a request share workgroups and tiles of its cache: what one of them
may not see yet reaches none of its bits, NaN and infinities too (mla_cache_attend)."""
import numpy as np
import pytest

import mx4_reference as R
from test_gpu_cache import _bf16_dev, _dev, own, random_cache, run_attend, table

pytestmark = pytest.mark.gpu

NQ = 5


def _spoil(raw, page, row, what):
    """Row `row` of a page of 64 rows: one group NaN, every group infinite (6 x 2^127 and -6 x 2^127 by
    its codes), a NaN or an infinite RoPE key."""
    if what == "nan group":
        raw[page, 64 * 256 + row * 16 + 9] = 255
    elif what == "infinite latent":
        raw[page, 64 * 256 + row * 16: 64 * 256 + row * 16 + 16] = 254
        raw[page, row * 256: row * 256 + 256] = 0xF7
    else:
        key = raw[page].view(np.uint16)[64 * 136 + row * 64: 64 * 136 + row * 64 + 64]
        key[3:50] = {"nan key": 0x7FC0, "infinite key": 0x7F80}[what]


# tokens that share a block of head-rows (all five; 3 and a part of the fourth), or have one of their own;
# a request over several workgroups, and batches whose requests lie within one
@pytest.mark.parametrize("heads", [3, 4, 6, 12, 20, 64, 128])
@pytest.mark.parametrize("seqs,keys", [(1, 150), (1, 66), (300, 68), (300, 40)])
@pytest.mark.parametrize("what", ["nan group", "infinite latent", "nan key", "infinite key"])
def test_a_later_token_reaches_no_earlier_one(heads, seqs, keys, what):
    import torch
    rng = np.random.default_rng(heads + keys)
    per = -(-keys // 64)
    raw = random_cache(rng, per, 64)
    pages, count = table([own(keys)], 64, rng.permutation(per))
    pages, count = np.tile(pages, (seqs, 1, 1)), np.tile(count, seqs)      # one cache for all requests
    pos = np.tile(np.arange(keys - NQ, keys, dtype=np.int32), (seqs, 1))
    pos[:, 1] = -1                                                        # a padded token among them
    q = rng.standard_normal((seqs, NQ, heads, 576)) * 0.5
    args = (_bf16_dev(q), _dev(pos), _dev(pages), _dev(count))
    clean, clean_lse = run_attend(R.geom(heads), *args, _dev(raw), 64)
    at = keys - 2                                                         # the position of token 3
    _spoil(raw, pages[0, at // 64, 0], at % 64, what)
    got, lse = run_attend(R.geom(heads), *args, _dev(raw), 64)
    for j in (0, 1, 2):
        assert torch.equal(got[:, j], clean[:, j]) and torch.equal(lse[:, j], clean_lse[:, j]), j
    assert torch.isfinite(clean).all()
    for j in (3, 4):
        if what in ("nan group", "nan key"):
            assert torch.isnan(got[:, j]).all() and torch.isnan(lse[:, j]).all(), j
        else:
            assert not torch.equal(got[:, j], clean[:, j]), j


def test_several_spoiled_keys_and_tiles():
    """Tokens in different tiles, each with its own NaN key: a token sees those up to its own."""
    import torch
    rng = np.random.default_rng(5)
    heads, keys = 8, 300
    raw = random_cache(rng, 5, 64)
    pages, count = table([own(keys)], 64, np.arange(5))
    pos = np.array([[63, 64, 120, 130, 290, 299]], dtype=np.int32)
    args = (_bf16_dev(rng.standard_normal((1, 6, heads, 576)) * 0.5), _dev(pos), _dev(pages), _dev(count))
    clean, clean_lse = run_attend(R.geom(heads), *args, _dev(raw), 64)
    for key in (125, 131, 200, 295):
        _spoil(raw, key // 64, key % 64, "nan group")
    got, lse = run_attend(R.geom(heads), *args, _dev(raw), 64)
    assert torch.equal(got[:, :3], clean[:, :3]) and torch.equal(lse[:, :3], clean_lse[:, :3])
    assert torch.isnan(got[:, 3:]).all() and torch.isnan(lse[:, 3:]).all()


@pytest.mark.parametrize("what", ["nan key", "infinite key", "infinite latent"])
def test_spoiled_keys_reach_only_their_request(what):
    """Keys that a request sees: the others of the batch, next to it in a workgroup, keep their bits."""
    import torch
    rng = np.random.default_rng(19)
    raw = random_cache(rng, 6, 64)
    lens = [100, 120, 64]
    pages, count = table([own(n) for n in lens], 64, np.arange(6))
    pos = np.array([[n - 1] for n in lens], dtype=np.int32)
    pages, count, pos = np.tile(pages, (100, 1, 1)), np.tile(count, 100), np.tile(pos, (100, 1))
    args = (_bf16_dev(rng.standard_normal((300, 1, 64, 576)) * 0.5), _dev(pos), _dev(pages), _dev(count))
    clean, clean_lse = run_attend(R.geom(64), *args, _dev(raw), 64)
    _spoil(raw, pages[1, 0, 0], 7, what)
    got, lse = run_attend(R.geom(64), *args, _dev(raw), 64)
    keep = torch.arange(300) % 3 != 1
    assert torch.equal(got[keep], clean[keep]) and torch.equal(lse[keep], clean_lse[keep])
    bad = ~torch.isfinite(lse[~keep])
    assert bad.all() if what == "nan key" else bad.any()
