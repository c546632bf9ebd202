"""GPU tests of the paged 4-bit latent cache (mla_cache_append, mla_cache_gather) and of the
attention over it (mla_cache_attend) against plain 64-bit definitions.  The tolerances are
the bounds that mx4_reference derives for each output."""
import numpy as np
import pytest

import mx4_reference as R

pytestmark = pytest.mark.gpu


def _dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _bf16_dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to(torch.bfloat16)


def _host(t):
    return t.float().cpu().numpy().astype(np.float64)


def random_cache(rng, pages, page_rows, lat=1.0, key=1.0):
    """A host cache of random rows, written by the definitions."""
    n = pages * page_rows
    c, s = R.quantize(R.bf16(rng.standard_normal((n, 512)) * lat))
    k = R.bf16(rng.standard_normal((n, 64)) * key).astype(np.float32).view(np.uint32) >> 16
    raw = np.concatenate((R.pack(c).reshape(pages, -1), s.astype(np.uint8).reshape(pages, -1),
                          k.astype(np.uint16).view(np.uint8).reshape(pages, -1)), 1)
    return np.ascontiguousarray(raw)


# ------------------------------------------------------------------ append, gather
@pytest.mark.parametrize("n,page_rows,stride,rotate", [(1, 64, 576, True), (3, 64, 584, False), (64, 128, 576, True), (70, 192, 640, True),
                                                       (501, 64, 2112, False), (1000, 256, 576, True), (0, 64, 576, True)])
def test_append_and_gather(n, page_rows, stride, rotate):
    import torch
    from paper_2609_07008_amd import mla
    rng = np.random.default_rng(n + stride)
    pages = n // page_rows + 3
    wide = rng.standard_normal((n, stride)) * 2.0 ** rng.integers(-6, 7, (1, stride))
    kv = _bf16_dev(wide)[:, :576] if n else torch.zeros((0, 576), dtype=torch.bfloat16, device="cuda")
    slots = rng.permutation(pages * page_rows)[:n].astype(np.int32)
    pos = rng.integers(-5, 1 << 20, n).astype(np.int32)
    if n > 2:
        pos[:2] = 0, 2 ** 31 - 1
    g = R.geom(64)
    before = rng.integers(0, 256, (pages, page_rows * 400), dtype=np.uint8)
    cache = _dev(before)
    mla.cache_append(g, kv, _dev(slots), cache, page_rows, pos=_dev(pos) if rotate else None)
    torch.cuda.synchronize()
    got = cache.cpu().numpy()
    x = _host(kv)
    c, s = R.quantize(x[:, :512]) if n else (np.zeros((0, 512), dtype=np.int64), np.zeros((0, 16), dtype=np.int64))

    def planes(raw):
        r = page_rows
        return (raw[:, : r * 256].reshape(-1, 256), raw[:, r * 256: r * 272].reshape(-1, 16),
                np.ascontiguousarray(raw[:, r * 272:]).view(np.uint16).reshape(-1, 64))
    codes, scales, rope = planes(got)
    assert np.array_equal(codes[slots], R.pack(c)) and np.array_equal(scales[slots], s)
    k = (rope[slots].astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    want = R.turned(x[:, 512:], pos) if rotate else x[:, 512:]
    if rotate:
        # half a bf16 step, and the sine's error (1.3e-7, the angle's own rounding 2e-7) on both terms
        both = np.abs(x[:, 512:]) + np.abs(np.roll(x[:, 512:], 32, 1))
        assert (np.abs(k - want) <= 2.0 ** -8 * np.abs(want) + 1e-6 * both).all()
    else:
        assert np.array_equal(k, want)
    others = np.ones(pages * page_rows, dtype=bool)
    others[slots] = False
    for a, b in zip(planes(got), planes(before)):
        assert np.array_equal(a[others], b[others])
    back = torch.full((n, stride), 3.0, dtype=torch.bfloat16, device="cuda")
    mla.cache_gather(g, _dev(slots), cache, page_rows, back[:, :576])
    torch.cuda.synchronize()
    y = _host(back)
    assert np.array_equal(y[:, :512], R.values(c, s)) and np.array_equal(y[:, 512:576], k) and (y[:, 576:] == 3).all()


def test_slots_outside_the_cache_are_skipped():
    import torch
    from paper_2609_07008_amd import mla
    rng = np.random.default_rng(2)
    kv = _bf16_dev(rng.standard_normal((6, 576)))
    before = random_cache(rng, 2, 64)
    cache = _dev(before)
    slots = _dev(np.array([-1, 128, 5, 2 ** 31 - 1, -2 ** 31, 127], dtype=np.int32))
    g = R.geom(8)
    mla.cache_append(g, kv, slots, cache, 64)
    out = torch.full((6, 576), 3.0, dtype=torch.bfloat16, device="cuda")
    mla.cache_gather(g, slots, cache, 64, out)
    torch.cuda.synchronize()
    got, y = cache.cpu().numpy(), _host(out)
    c, s = R.quantize(_host(kv)[:, :512])
    for i, slot in ((2, 5), (5, 127)):
        assert np.array_equal(got[slot // 64, slot % 64 * 256: slot % 64 * 256 + 256], R.pack(c)[i])
        assert np.array_equal(y[i, :512], R.values(c, s)[i])
    changed = (got != before)
    assert set(np.nonzero(changed)[0]) <= {0, 1} and changed.sum() <= 2 * 400
    assert (y[[0, 1, 3, 4]] == 3).all()


def test_gather_repeated_slots():
    import torch
    from paper_2609_07008_amd import mla
    rng = np.random.default_rng(6)
    raw = random_cache(rng, 1, 64)
    slots = np.array([9, 9, 9, 0, 63, 9], dtype=np.int32)
    out = torch.empty((6, 576), dtype=torch.bfloat16, device="cuda")
    mla.cache_gather(R.geom(8), _dev(slots), _dev(raw), 64, out)
    lat, key = R.Cache(raw, 64).rows(0)
    assert np.array_equal(_host(out), np.concatenate((lat, key), 1)[slots])


# ------------------------------------------------------------------ attention
def run_attend(g, q, pos, pages, seq_pages, cache, page_rows, lse=True, ws=None):
    import torch
    from paper_2609_07008_amd import mla
    b, nq, heads, _ = q.shape
    out = torch.full((b, nq, heads, 512), float("nan"), dtype=torch.bfloat16, device="cuda")
    out_lse = torch.full((b, nq, heads), float("nan"), dtype=torch.float32, device="cuda") if lse else None
    if ws is None:
        ws = torch.full((mla.cache_attend_query(g, b, nq, pages.shape[1], page_rows),), 0xFF, dtype=torch.uint8, device="cuda")
    mla.cache_attend(g, q, pos, pages, seq_pages, cache, page_rows, out, out_lse, workspace=ws)
    torch.cuda.synchronize()
    return out, out_lse


def table(requests, page_rows, ids, max_pages=None):
    """pages [B, max, 4] and seq_pages of requests: lists of segments (request position, rows, frame, open)."""
    lists = []
    at = 0
    for segs in requests:
        e = []
        for p0, rows, frame, is_open in segs:
            for u in range(0, rows, page_rows):
                e.append((ids[at], page_rows if is_open else min(page_rows, rows - u), p0 + u, frame))
                at += 1
        lists.append(e)
    most = max_pages or max(1, max(len(e) for e in lists))
    t = np.full((len(lists), most, 4), -7, dtype=np.int32)
    for b, e in enumerate(lists):
        t[b, : len(e)] = np.array(e, dtype=np.int32).reshape(-1, 4)
    return t, np.array([len(e) for e in lists], dtype=np.int32)


def check_attend(g, q, pos, pages, seq_pages, raw, page_rows, tag=""):
    qd = _bf16_dev(q)
    out, lse = run_attend(g, qd, _dev(pos), _dev(pages), _dev(seq_pages), _dev(raw), page_rows)
    want, want_lse, b_out, b_lse = R.attend(g, _host(qd), pos, pages, seq_pages, R.Cache(raw, page_rows))
    o, l = _host(out), lse.cpu().numpy().astype(np.float64)
    empty = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(l), empty), tag
    assert (o[empty] == 0).all(), tag
    assert np.isfinite(o).all() and (np.abs(o - want) <= b_out).all(), (tag, np.abs(o - want).max(), b_out.max())
    d = np.abs(l[~empty] - want_lse[~empty])
    assert (d <= b_lse[~empty]).all(), (tag, d.max(), b_lse.max())
    return out, lse


def own(n):
    return [(0, n, 0, True)]


CASES = {
    # heads, n_q, page_rows, lengths of plain requests (keys 0 .. n - 1, one token at n - 1)
    "one_key": (64, 1, 64, [1]),
    "few": (1, 1, 64, [1, 2, 63, 64, 65]),
    "share_of_heads": (16, 1, 64, [127, 128, 129, 500, 1, 40]),
    "eight_heads_wide_pages": (8, 1, 256, [300, 257, 256, 255]),
    "thirty_three_head_rows": (33, 1, 128, [200, 77]),
    "twenty_heads_three_tokens": (20, 3, 64, [130, 64, 3, 2, 1]),
    "sixty_four": (64, 1, 64, [1000, 333, 64]),
    "one_hundred_twenty_eight": (128, 1, 192, [260, 191]),
    "five_tokens": (64, 5, 64, [70, 200, 5]),
    "long": (64, 1, 64, [9000]),
}


@pytest.mark.parametrize("name", sorted(CASES))
def test_attend_plain_requests(name):
    heads, nq, pr, lens = CASES[name]
    rng = np.random.default_rng(len(name))
    need = sum(-(-n // pr) for n in lens)
    raw = random_cache(rng, need + 2, pr)
    pages, count = table([own(n) for n in lens], pr, rng.permutation(need + 2))
    pos = np.array([[n - nq + j for j in range(nq)] for n in lens], dtype=np.int32)   # may start below 0
    q = rng.standard_normal((len(lens), nq, heads, 576)) * 0.5
    check_attend(R.geom(heads), q, pos, pages, count, raw, pr, name)


@pytest.mark.parametrize("heads,nq", [(128, 20), (128, 66), (96, 3)])
def test_attend_many_head_rows(heads, nq):
    """Shares of many head-row blocks, fewer than the XCDs or not a multiple of them."""
    rng = np.random.default_rng(nq)
    lens = [150, nq]
    raw = random_cache(rng, 8, 64)
    pages, count = table([own(n) for n in lens], 64, rng.permutation(8))
    pos = np.array([[n - nq + j for j in range(nq)] for n in lens], dtype=np.int32)
    check_attend(R.geom(heads), rng.standard_normal((2, nq, heads, 576)) * 0.5, pos, pages, count, raw, 64)


@pytest.mark.parametrize("heads,nq,pr", [(64, 1, 64), (16, 2, 128), (128, 1, 64)])
def test_attend_relocated_documents(heads, nq, pr):
    """Documents in their canonical frames at far request positions, stored in any order and
    ending inside pages; one shared by two requests at different places."""
    rng = np.random.default_rng(heads)
    raw = random_cache(rng, 40, pr, key=2.0)
    ids = rng.permutation(40)
    segs = [[(90, 130, 90, False), (0, 90, 0, False), (100000, 65, 100000, False), (262000, 100, 0, True)],
            [(0, 1, 0, False), (1, 70, 1, False), (71, 33, 0, True)]]
    pages, count = table(segs, pr, ids)
    pages[1, 1] = pages[0, 0]              # the shared document's first page
    pages[1, 1, 2:] = 1, 1
    pos = np.stack((np.arange(nq) + 262050, np.arange(nq) + 95)).astype(np.int32)
    q = rng.standard_normal((2, nq, heads, 576))
    check_attend(R.geom(heads), q, pos, pages, count, raw, pr)


def test_attend_a_document_answers_alike_wherever_it_lies():
    """A request moved as a whole by any offset has the same scores: same output bits up to the
    rounding of the angles."""
    rng = np.random.default_rng(31)
    raw = random_cache(rng, 8, 64)
    q = rng.standard_normal((1, 1, 64, 576))
    got = []
    for off in (0, 12345, 2 ** 30):
        pages, count = table([[(off, 200, off, False), (off + 200, 60, off + 200, True)]], 64, np.arange(8))
        pos = np.array([[off + 255]], dtype=np.int32)
        got.append(check_attend(R.geom(64), q, pos, pages, count, raw, 64, str(off))[0])
    import torch
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_attend_odd_entries():
    """Entries that hold nothing or lie outside the cache, counts outside the table, padded
    tokens, a request without pages: each as if those keys were not there."""
    rng = np.random.default_rng(4)
    raw = random_cache(rng, 6, 64)
    pages = np.zeros((5, 4, 4), dtype=np.int32)
    pages[0] = [(0, 64, 0, 0), (-1, 64, 64, 0), (6, 64, 64, 0), (1, 10, 64, 0)]
    pages[1] = [(2, -5, 0, 0), (2, 0, 0, 0), (3, 1000, 0, 0), (2 ** 31 - 1, 64, 0, 0)]
    pages[2] = [(4, 64, -30, 0), (5, 64, 34, 0), (0, 64, 2 ** 31 - 1, 0), (1, 64, -2 ** 31, 0)]
    pages[3] = [(0, 64, 0, 0), (1, 64, 64, 0), (2, 64, 128, 0), (3, 64, 192, 0)]
    pages[4] = pages[3]
    count = np.array([4, 9, 4, 0, -3], dtype=np.int32)
    pos = np.array([[70, -1], [63, 20], [40, 0], [100, 100], [5, 5]], dtype=np.int32)
    q = rng.standard_normal((5, 2, 16, 576)) * 0.5
    check_attend(R.geom(16), q, pos, pages, count, raw, 64)
    pos[:] = -1
    check_attend(R.geom(16), q, pos, pages, count, raw, 64)


@pytest.mark.parametrize("heads", [16, 64])
def test_attend_unwritten_rows_hold_anything(heads):
    """NaN scales, NaN and infinite RoPE keys behind a page's rows, past the last position and
    in pages allocated ahead."""
    rng = np.random.default_rng(heads + 1)
    raw = random_cache(rng, 7, 64)
    clean = raw.copy()

    def spoil(page, lo):
        raw[page, lo * 256: 64 * 256] = 0xFF
        raw[page, 64 * 256 + lo * 16: 64 * 272] = 255
        raw[page].view(np.uint16)[64 * 136 + lo * 64:] = rng.choice([0x7FC0, 0x7F80, 0xFF80], (64 - lo) * 64)
    spoil(1, 40)
    spoil(3, 11)
    spoil(4, 0)
    pages = np.array([[(0, 64, 0, 0), (1, 40, 64, 64), (2, 64, 104, 0), (3, 64, 168, 0), (4, 64, 232, 0)],
                      [(5, 64, 0, 0), (3, 11, 64, 0), (4, 0, 75, 0), (-1, 64, 75, 0), (6, 64, 75, 0)]], dtype=np.int32)
    count = np.array([5, 5], dtype=np.int32)
    pos = np.array([[178], [90]], dtype=np.int32)
    q = rng.standard_normal((2, 1, heads, 576)) * 0.5
    a = check_attend(R.geom(heads), q, pos, pages, count, raw, 64)
    b = run_attend(R.geom(heads), _bf16_dev(q), _dev(pos), _dev(pages), _dev(count), _dev(clean), 64)
    import torch
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_attend_rising_scores():
    """Scores that rise from tile to tile by more than the softmax reference allows, fall
    again, and differ by hundreds between head-rows."""
    rng = np.random.default_rng(77)
    pr, n = 64, 640
    lat = rng.standard_normal((n, 512)) * 0.05
    u = rng.standard_normal(512)
    u /= np.linalg.norm(u)
    level = np.concatenate((np.linspace(-300, 900, 400), np.linspace(900, -500, 240)))
    lat += level[:, None] * u / 20
    c, s = R.quantize(R.bf16(lat))
    raw = random_cache(rng, n // pr, pr)
    raw[:, : pr * 256] = R.pack(c).reshape(n // pr, -1)
    raw[:, pr * 256: pr * 272] = s.astype(np.uint8).reshape(n // pr, -1)
    q = rng.standard_normal((1, 1, 64, 576)) * 0.05
    q[0, 0, :, :512] += np.linspace(-80, 80, 64)[:, None] * u
    pages, count = table([own(n)], pr, np.arange(n // pr))
    check_attend(R.geom(64), q, np.array([[n - 1]], dtype=np.int32), pages, count, raw, pr)


def test_attend_nan_and_infinite_keys_reach_only_their_request():
    import torch
    rng = np.random.default_rng(9)
    raw = random_cache(rng, 6, 64)
    pages, count = table([own(100), own(120), own(64)], 64, np.arange(6))
    pos = np.array([[99], [119], [63]], dtype=np.int32)
    q = rng.standard_normal((3, 1, 64, 576)) * 0.5
    args = (_dev(pos), _dev(pages), _dev(count))
    clean, clean_lse = run_attend(R.geom(64), _bf16_dev(q), *args, _dev(raw), 64)
    raw[2, 64 * 256 + 7 * 16 + 3] = 255                        # a NaN group in the second request
    got, lse = run_attend(R.geom(64), _bf16_dev(q), *args, _dev(raw), 64)
    assert torch.isnan(got[1]).all() and torch.isnan(lse[1]).all()
    for b in (0, 2):
        assert torch.equal(got[b], clean[b]) and torch.equal(lse[b], clean_lse[b])


@pytest.mark.parametrize("seqs", [1, 513, 1500])
def test_attend_many_requests(seqs):
    """Batches below and above the scan's width; lengths 0 .. 130."""
    rng = np.random.default_rng(seqs)
    lens = rng.integers(0, 131, seqs)
    lens[0] = 130
    need = int(sum(-(-n // 64) for n in lens))
    raw = random_cache(rng, need, 64)
    pages, count = table([own(n) if n else [] for n in lens], 64, rng.permutation(need))
    pos = (lens[:, None] - 1).astype(np.int32)
    q = rng.standard_normal((seqs, 1, 4, 576)) * 0.5
    check_attend(R.geom(4), q, pos, pages, count, raw, 64)


@pytest.mark.parametrize("heads", [4, 64])
def test_attend_batch_with_holes(heads):
    """A few requests far apart in a padded batch, several of them in one workgroup's share."""
    rng = np.random.default_rng(heads)
    lens = np.zeros(1300, dtype=np.int64)
    lens[[3, 66, 67, 400, 831, 1299]] = 130, 64, 1, 200, 65, 700
    need = int(sum(-(-n // 64) for n in lens))
    raw = random_cache(rng, need, 64)
    pages, count = table([own(n) if n else [] for n in lens], 64, rng.permutation(need))
    pos = (lens[:, None] - 1).astype(np.int32)
    check_attend(R.geom(heads), rng.standard_normal((1300, 1, heads, 576)) * 0.5, pos, pages, count, raw, 64)


def test_attend_batch_of_none_and_without_pages():
    import torch
    from paper_2609_07008_amd import mla
    g = R.geom(8)
    cache = torch.zeros((1, 64 * 400), dtype=torch.uint8, device="cuda")
    for b, most in ((0, 3), (2, 0)):
        q = torch.ones((b, 1, 8, 576), dtype=torch.bfloat16, device="cuda")
        out, lse = run_attend(g, q, torch.zeros((b, 1), dtype=torch.int32, device="cuda"),
                              torch.zeros((b, most, 4), dtype=torch.int32, device="cuda"),
                              torch.full((b,), 5, dtype=torch.int32, device="cuda"), cache, 64)
        assert (out == 0).all() and torch.isneginf(lse).all()


def test_attend_offsets_past_32_bits():
    """A cache of over 2^32 bytes whose last pages are used, and the same rows at its start."""
    import torch
    from paper_2609_07008_amd import mla
    rng = np.random.default_rng(1)
    pr, pages_n = 64, 180000                                   # 4.6 GB
    cache = torch.zeros((pages_n, pr * 400), dtype=torch.uint8, device="cuda")
    kv = _bf16_dev(rng.standard_normal((300, 576)))
    g = R.geom(64)
    lo = torch.arange(300, dtype=torch.int32, device="cuda")
    hi = lo + (pages_n - 5) * pr
    q = _bf16_dev(rng.standard_normal((1, 1, 64, 576)))
    pos = torch.tensor([[290]], dtype=torch.int32, device="cuda")
    count = torch.tensor([5], dtype=torch.int32, device="cuda")
    got = []
    for first, slots in ((0, lo), (pages_n - 5, hi)):
        mla.cache_append(g, kv, slots, cache, pr, pos=lo)
        back = torch.empty_like(kv)
        mla.cache_gather(g, slots, cache, pr, back)
        p = torch.tensor([[(first + i, pr, i * pr, 0) for i in range(5)]], dtype=torch.int32, device="cuda")
        got.append((back, *run_attend(g, q, pos, p, count, cache, pr)))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    small = cache[pages_n - 5:].cpu().numpy()
    p = np.array([[(i, pr, i * pr, 0) for i in range(5)]], dtype=np.int32)
    check_attend(g, _host(q), pos.cpu().numpy(), p, np.array([5], dtype=np.int32), small, pr)


def test_attend_without_lse_and_twice_the_same_bits():
    import torch
    rng = np.random.default_rng(21)
    raw = _dev(random_cache(rng, 30, 64))
    pages, count = table([own(700), own(900)], 64, np.arange(30))
    args = (_bf16_dev(rng.standard_normal((2, 1, 64, 576))), _dev(np.array([[699], [899]], dtype=np.int32)), _dev(pages), _dev(count))
    a, lse = run_attend(R.geom(64), *args, raw, 64)
    for _ in range(3):
        b, none = run_attend(R.geom(64), *args, raw, 64, lse=False)
        assert none is None and torch.equal(a, b)
