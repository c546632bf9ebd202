"""Batches of mla_cache_attend in which a few requests hold most of the keys: many shares of
the work to join for them, one or two for the others, in one call."""
import numpy as np
import pytest

import mx4_reference as R
from test_gpu_cache import _bf16_dev, _dev, _host, check_attend, own, random_cache, run_attend, table

pytestmark = pytest.mark.gpu

# heads, n_q, requests, {request: keys} of the long ones, keys of the others (0 .. this)
CASES = {
    "one_first": (16, 1, 64, {0: 9000}, 130),
    "one_last": (64, 1, 70, {69: 12800}, 64),
    "one_among_empty": (16, 1, 200, {77: 16000}, 0),
    "two_that_meet": (32, 1, 64, {30: 5000, 31: 6000}, 200),
    "several_lengths": (16, 1, 64, {3: 2400, 20: 600, 21: 530, 40: 64, 41: 9000, 63: 1100}, 70),
    "around_thirty_two_shares": (4, 1, 300, {7: 33 * 64, 9: 32 * 64, 100: 34 * 64, 299: 65 * 64}, 0),
    "around_nine_shares": (4, 1, 300, {7: 9 * 64, 9: 8 * 64, 100: 10 * 64, 299: 17 * 64}, 64),
    "runs_of_three_tokens": (64, 3, 40, {11: 7000, 12: 3000}, 100),
    "four_blocks": (128, 2, 20, {5: 6000, 19: 4000}, 200),
    "seven_shares": (66, 32, 8, {2: 3000}, 64),
    "thirty_six_shares": (64, 7, 12, {0: 200, 4: 9000}, 0),
}


@pytest.mark.parametrize("name", sorted(CASES))
def test_skewed_batch(name):
    heads, nq, seqs, long, rest = CASES[name]
    rng = np.random.default_rng(len(name))
    lens = rng.integers(0, rest + 1, seqs)
    for b, n in long.items():
        lens[b] = n
    need = int(sum(-(-n // 64) for n in lens))
    raw = random_cache(rng, need, 64)
    pages, count = table([own(n) if n else [] for n in lens], 64, rng.permutation(need))
    pos = (lens[:, None] - nq + np.arange(nq)[None]).astype(np.int32)
    check_attend(R.geom(heads), rng.standard_normal((seqs, nq, heads, 576)) * 0.5, pos, pages, count, raw, 64, name)


def test_a_request_answers_alike_at_every_place():
    """One long request before, between and behind 80 empty ones: the same runs of tiles, so the
    same bits."""
    import torch
    rng = np.random.default_rng(2)
    n, seqs = 40 * 64, 81
    raw = _dev(random_cache(rng, 40, 64))
    q = rng.standard_normal((1, 1, 16, 576))
    want = None
    for place in (0, 1, 7, 40, 63, 64, 79, 80):
        pages, count = table([own(n) if b == place else [] for b in range(seqs)], 64, np.arange(40))
        pos = np.where(np.arange(seqs) == place, n - 1, -1)[:, None].astype(np.int32)
        out, lse = run_attend(R.geom(16), _bf16_dev(np.tile(q, (seqs, 1, 1, 1))), _dev(pos), _dev(pages), _dev(count), raw, 64)
        others = torch.arange(seqs) != place
        assert (out[others] == 0).all() and torch.isneginf(lse[others]).all()
        got = (out[place].clone(), lse[place].clone())
        want = want or got
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), place


@pytest.mark.parametrize("seqs", [65471, 65480, 65535])
def test_long_request_in_the_largest_batches(seqs):
    """As many requests as a call takes, and one of 100 tiles among them."""
    rng = np.random.default_rng(seqs)
    n, place = 6350, 40000
    raw = random_cache(rng, 100, 64)
    pages = np.zeros((seqs, 100, 4), dtype=np.int32)
    pages[place], count = table([own(n)], 64, rng.permutation(100))[0][0], np.zeros(seqs, dtype=np.int32)
    count[place] = 100
    pos = np.full((seqs, 1), -1, dtype=np.int32)
    pos[place] = n - 1
    check_attend(R.geom(2), np.broadcast_to(rng.standard_normal((1, 1, 2, 576)) * 0.5, (seqs, 1, 2, 576)), pos, pages, count, raw, 64)
