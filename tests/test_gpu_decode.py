"""GPU tests of a decode layer on the paged 4-bit cache (step.DecodeStep: append, attend,
o-proj over all heads, 4-bit W_b) against the chained 64-bit definitions, and as a serving
loop uses it: captured once and replayed, on other streams, two at a time, with padded
requests.  Bounds are carried from each output into the next."""
import numpy as np
import pytest

import mx4_reference as R
from test_gpu_cache import _bf16_dev, _dev, _host, check_attend, random_cache, run_attend, table

pytestmark = pytest.mark.gpu


def _layer(rng, g, d_out):
    """W_o [n_pg, H/n_pg * 512, d_model/n_pg] bf16, W_b [d_out, d_model] as codes and scales."""
    npg = g.n_proj_groups
    w_o = _bf16_dev(rng.standard_normal((npg, g.n_heads // npg * 512, g.d_model // npg)) / 64)
    c, s = R.quantize(R.bf16(rng.standard_normal((d_out, g.d_model)) / 16))
    return w_o, c, s


def _batch(rng, g, n_q, page_rows, most):
    """Four requests over a random cache: one in the middle of a page, one behind two documents
    in their own frames, one with only its new tokens, one padded.  Returns the arguments that a
    step takes, as host arrays."""
    heads = g.n_heads
    lens = (page_rows + 31, 40, 0)
    ids = rng.permutation(12)
    pages, count = table([[(0, lens[0] + n_q, 0, True)],
                          [(7, 90, 7, False), (0, 7, 0, False), (97, lens[1] + n_q, 97, True)],
                          [(0, n_q, 0, True)], []], page_rows, ids, most)
    first = (lens[0], 97 + lens[1], 0)
    pos = np.full((4, n_q), -1, dtype=np.int32)
    slots = np.full((4, n_q), -1, dtype=np.int32)
    turn = np.zeros((4, n_q), dtype=np.int32)
    for b in range(3):
        for j in range(n_q):
            t = first[b] + j
            e = [e for e in pages[b, : count[b]] if e[2] <= t < e[2] + page_rows][-1]
            pos[b, j], slots[b, j], turn[b, j] = t, e[0] * page_rows + t - e[2], t - e[3]
    return dict(kv=rng.standard_normal((4 * n_q, 576)), q=rng.standard_normal((4, n_q, heads, 576)) * 0.5, pos=pos,
                slots=slots.reshape(-1), turn=turn.reshape(-1), pages=pages, seq_pages=count)


def _upload(a):
    return {k: _bf16_dev(v) if v.dtype.kind == "f" else _dev(v) for k, v in a.items()}


def _run(st, d, cache, layer, stream=None):
    w_o, codes, scales = layer
    return st.run(d["kv"], d["slots"], d["q"], d["pos"], d["pages"], d["seq_pages"], cache, w_o, codes, scales, turn=d["turn"],
                  stream=stream)


def _codes_dev(c, s):
    return _dev(R.pack(c)), _dev(s.astype(np.uint8))


@pytest.mark.parametrize("heads,n_q,page_rows,npg,d_out", [(16, 1, 64, 1, 203), (64, 2, 128, 4, 320), (128, 1, 64, 2, 33)])
def test_decode_step(heads, n_q, page_rows, npg, d_out):
    import torch
    from paper_2609_07008_amd.step import DecodeStep
    rng = np.random.default_rng(heads + n_q)
    g = R.geom(heads, n_proj_groups=npg)
    w_o, c, s = _layer(rng, g, d_out)
    a = _batch(rng, g, n_q, page_rows, 5)
    raw = random_cache(rng, 12, page_rows)
    cache = _dev(raw)
    st = DecodeStep(g, 4, n_q, 5, page_rows, d_out, y_dtype=torch.float32, with_lse=True)
    d = _upload(a)
    y = _host(_run(st, d, cache, (w_o, *_codes_dev(c, s))))
    got = R.Cache(cache.cpu().numpy(), page_rows)
    kv = _host(d["kv"])
    kc, ks = R.quantize(kv[:, :512])
    for i, slot in enumerate(a["slots"]):
        if slot >= 0:
            assert np.array_equal(got.rows(slot // page_rows)[0][slot % page_rows], R.values(kc[i: i + 1], ks[i: i + 1])[0])
    o, lse, b_o, b_lse = R.attend(g, _host(d["q"]), a["pos"], a["pages"], a["seq_pages"], got)
    empty = np.isneginf(lse)
    assert (np.abs(_host(st.out_o) - o) <= b_o).all()
    # z: heads * 512 products in 32-bit sums of bf16 head outputs, rounded to bf16
    n, per = 4 * n_q, heads // npg
    w = _host(w_o)
    oo, bo = o.reshape(n, npg, per * 512), b_o.reshape(n, npg, per * 512)
    z = np.concatenate([oo[:, p] @ w[p] for p in range(npg)], 1)
    mag = np.concatenate([np.abs(oo[:, p]) @ np.abs(w[p]) for p in range(npg)], 1)
    b_z = np.concatenate([bo[:, p] @ np.abs(w[p]) for p in range(npg)], 1)
    b_z += per * 512 * 2.0 ** -24 * (mag + b_z)
    b_z += 2.0 ** -8 * (np.abs(z) + b_z)
    zk = _host(st.z)
    assert (np.abs(zk - z) <= b_z).all()
    wb = R.values(c, s)
    b_y = b_z @ np.abs(wb).T + g.d_model * 2.0 ** -24 * ((np.abs(z) + b_z) @ np.abs(wb).T)
    assert (np.abs(y - z @ wb.T) <= b_y).all()
    assert (y[3 * n_q:] == 0).all() and empty[3].all()      # the padded request


def test_decode_step_captured_and_replayed():
    """One capture; positions, slots, pages, queries and rows change between the replays, with
    eager calls and synchronizations between.  Every replay gives the eager bits."""
    import torch
    from paper_2609_07008_amd.step import DecodeStep
    rng = np.random.default_rng(3)
    g = R.geom(64)
    w_o, c, s = _layer(rng, g, 96)
    layer = (w_o, *_codes_dev(c, s))
    raw = _dev(random_cache(rng, 12, 64))
    steps = [_upload(_batch(rng, g, 1, 64, 5)) for _ in range(5)]
    eager, cap = (DecodeStep(g, 4, 1, 5, 64, 96, with_lse=True) for _ in range(2))
    live = {k: v.clone() for k, v in steps[0].items()}
    cache = raw.clone()
    _run(cap, live, cache, layer)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _run(cap, live, cache, layer)
    for i in (1, 2, 3, 4, 0):
        want_cache = raw.clone()
        want = [t.clone() for t in (_run(eager, steps[i], want_cache, layer), eager.out_o, eager.out_lse)]
        for k in live:
            live[k].copy_(steps[i][k])
        cache.copy_(raw)
        for t in (cap.y, cap.out_o, cap.out_lse, cap.z):
            t.fill_(float("nan"))
        cap.ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip((cap.y, cap.out_o, cap.out_lse), want):
            assert torch.equal(got, ref), i
        assert torch.equal(cache, want_cache), i


def test_two_steps_at_once_on_their_own_streams():
    import torch
    from paper_2609_07008_amd.step import DecodeStep
    rng = np.random.default_rng(8)
    g = R.geom(64)
    w_o, c, s = _layer(rng, g, 128)
    layer = (w_o, *_codes_dev(c, s))
    raws = [_dev(random_cache(rng, 12, 64)) for _ in range(2)]
    args = [_upload(_batch(rng, g, 2, 64, 5)) for _ in range(2)]
    steps = [DecodeStep(g, 4, 2, 5, 64, 128, with_lse=True) for _ in range(2)]
    want = []
    for st, d, raw in zip(steps, args, raws):
        cache = raw.clone()
        want.append([t.clone() for t in (_run(st, d, cache, layer), st.out_o, st.out_lse, cache)])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    caches = [r.clone() for r in raws]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, d, cache, stream in zip(steps, args, caches, streams):
            _run(st, d, cache, layer, stream)
    torch.cuda.synchronize()
    for st, cache, w in zip(steps, caches, want):
        for got, ref in zip((st.y, st.out_o, st.out_lse, cache), w):
            assert torch.equal(got, ref)


def test_gathered_document_in_the_online_attention():
    """A document appended in its own frame, gathered back and attended by mla_online_attend,
    next to mla_cache_attend on the pages: one answer, and that of the definitions."""
    import torch
    from paper_2609_07008_amd import mla
    from paper_2609_07008_amd.step import OnlineStep
    rng = np.random.default_rng(12)
    heads, n, pr, off = 4, 100, 64, 5000
    g = R.geom(heads, n_groups=heads)
    kv = _bf16_dev(rng.standard_normal((n, 576)))
    cache = torch.zeros((3, pr * 400), dtype=torch.uint8, device="cuda")
    slots = torch.arange(n, dtype=torch.int32, device="cuda") + pr
    mla.cache_append(g, kv, slots, cache, pr)
    back = torch.empty_like(kv)
    mla.cache_gather(g, slots, cache, pr, back)
    q = rng.standard_normal((1, n, heads, 576)) * 0.5
    # the document alone, and far on in a request: the same relative positions
    st = OnlineStep(g, [(0, n, 0)], np.zeros(0, dtype=np.int32), np.zeros(heads, dtype=np.int32), 0)
    qd = _bf16_dev(q)
    st.attend(back, qd[0], None)
    st.merge()
    pages = np.array([[(1, 64, off, off), (2, n - 64, off + 64, off)]], dtype=np.int32)
    pos = (off + np.arange(n, dtype=np.int32))[None]
    out, _ = check_attend(g, q, pos, pages, np.array([2], dtype=np.int32), cache.cpu().numpy(), pr)
    want, _, b_o, _ = R.attend(g, _host(qd), pos, pages, np.array([2], dtype=np.int32), R.Cache(cache.cpu().numpy(), pr))
    # mla_online_attend rounds the turned query to bf16 once: a score is off by up to a half
    # step of each RoPE product, and the output by twice that of the largest value
    x = np.abs(_host(qd)[0, :, :, 512:])
    lat, key = _host(back)[:, :512], _host(back)[:, 512:]
    pair = x + np.roll(x, 32, -1)
    d = 2.0 ** -8 * (pair @ np.abs(key).T).max(-1) * g.softmax_scale
    b = b_o[0] + 2 * np.expm1(d)[..., None] * np.abs(lat).max()
    assert (np.abs(_host(st.out_o).reshape(n, heads, 512) - want[0]) <= b).all()


@pytest.mark.parametrize("heads", [8, 16, 24, 32])
def test_references_that_differ_between_score_waves(heads):
    """Up to 32 head-rows the keys of a tile are scored by several waves: scores that rise and
    fall within a tile by more than the softmax reference allows, some waves without a key."""
    rng = np.random.default_rng(heads)
    pr, n = 64, 330
    u = rng.standard_normal(512)
    u /= np.linalg.norm(u)
    level = 40 * np.sin(np.arange(n) * 0.9) * np.linspace(0, 20, n)
    c, s = R.quantize(R.bf16(rng.standard_normal((n, 512)) * 0.05 + level[:, None] * u / 20))
    full = -(-n // pr)
    raw = random_cache(rng, full, pr)
    codes = np.zeros((full * pr, 256), dtype=np.uint8)
    scales = np.full((full * pr, 16), 127, dtype=np.uint8)
    codes[:n], scales[:n] = R.pack(c), s
    raw[:, : pr * 256] = codes.reshape(full, -1)
    raw[:, pr * 256: pr * 272] = scales.reshape(full, -1)
    q = rng.standard_normal((3, 1, heads, 576)) * 0.05
    q[:, 0, :, :512] += np.linspace(-40, 40, heads)[:, None] * u
    pages, count = table([[(0, n, 0, True)]] * 3, pr, list(range(full)) * 3)
    pos = np.array([[n - 1], [17], [64]], dtype=np.int32)
    check_attend(R.geom(heads), q, pos, pages, count, raw, pr)


@pytest.mark.parametrize("heads", [4, 24, 64])
def test_a_request_of_nan_keys_alone(heads):
    """Nothing but NaN scores, in one tile and over several workgroups: NaN, not an empty row."""
    import torch
    rng = np.random.default_rng(heads)
    raw = random_cache(rng, 6, 64)
    raw[:5, 64 * 256: 64 * 272] = 255
    pages, count = table([[(0, 1, 0, True)], [(0, 70, 0, True)], [(0, 128, 0, True)], [(0, 64, 0, True)]], 64, [0, 1, 2, 3, 4, 5])
    pos = np.array([[0], [69], [127], [63]], dtype=np.int32)
    q = rng.standard_normal((4, 1, heads, 576)) * 0.5
    out, lse = run_attend(R.geom(heads), _bf16_dev(q), _dev(pos), _dev(pages), _dev(count), _dev(raw), 64)
    assert torch.isnan(out[:3]).all() and torch.isnan(lse[:3]).all()
    assert torch.isfinite(out[3]).all() and torch.isfinite(lse[3]).all()


@pytest.mark.parametrize("heads,n", [(4, 1), (64, 1), (24, 90), (64, 200)])
def test_one_value_is_answered_exactly(heads, n):
    """A request of one key, or of keys with one latent: the output is that latent, whatever the
    weights and their rounding (its bf16 values are exact); over several workgroups too."""
    import torch
    from paper_2609_07008_amd import mla
    rng = np.random.default_rng(n + heads)
    raw = random_cache(rng, 4, 64)
    raw[:, : 64 * 256] = np.tile(raw[0, :256], (4, 64))
    raw[:, 64 * 256: 64 * 272] = np.tile(raw[0, 64 * 256: 64 * 256 + 16], (4, 64))
    pages, count = table([[(0, n, 0, True)]], 64, [0, 1, 2, 3])
    q = _bf16_dev(rng.standard_normal((1, 1, heads, 576)))
    out, _ = run_attend(R.geom(heads), q, _dev(np.array([[n - 1]], dtype=np.int32)), _dev(pages), _dev(count), _dev(raw), 64)
    lat, _ = R.Cache(raw, 64).rows(0)
    want = np.broadcast_to(lat[0], (heads, 512))
    got = _host(out)[0, 0]
    # sums of n terms w v and n terms w in 32 bits, one division, one rounding to bf16: next to
    # an exact bf16 value the 32-bit errors (n 2^-24 each) do not reach half a bf16 step
    assert np.array_equal(got, want)
