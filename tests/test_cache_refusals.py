"""What the 4-bit and cache entry points refuse, on the host before any device work (CPU):
the C ABI's checks with made-up addresses, and the binding's checks of tensors."""
import ctypes

import numpy as np
import pytest

import mx4_reference as R

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 6
A = 4096   # an aligned address that is never read


@pytest.fixture(scope="module")
def mla():
    from paper_2609_07008_amd import mla as m
    return m


def _p(v):
    return None if v is None else ctypes.c_void_p(v)


QUANT = dict(n=2, c=64, x=A, stride=64, codes=A, scales=A)


@pytest.mark.parametrize("over,status", [
    (dict(n=-1), SHAPE), (dict(c=0), SHAPE), (dict(c=48), SHAPE), (dict(stride=56), SHAPE), (dict(stride=68), SHAPE),
    (dict(x=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(x=A + 8), SHAPE), (dict(codes=A + 4), SHAPE),
    (dict(n=2 ** 62), SHAPE), (dict(n=0, x=None, codes=None, scales=None), OK)])
def test_quantize_refusals(mla, over, status):
    d = {**QUANT, **over}
    assert mla.LIB.mla_mx4_quantize(d["n"], d["c"], _p(d["x"]), d["stride"], _p(d["codes"]), _p(d["scales"]), None) == status
    assert mla.LIB.mla_mx4_dequantize(d["n"], d["c"], _p(d["codes"]), _p(d["scales"]), _p(d["x"]), d["stride"], None) == status
    assert (mla.LIB.mla_last_error_detail() == b"") == (status == OK)


WB = dict(n=2, d_in=128, d_out=8, z=A, codes=A, scales=A, out=1, y=A)


@pytest.mark.parametrize("over,status", [
    (dict(n=-1), SHAPE), (dict(n=1025), UNSUPPORTED), (dict(d_in=0), SHAPE), (dict(d_in=96), SHAPE), (dict(d_in=16448), UNSUPPORTED),
    (dict(d_out=0), SHAPE), (dict(d_out=2 ** 31 - 1), UNSUPPORTED), (dict(out=2), SHAPE), (dict(z=None), NULL),
    (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(y=None), NULL), (dict(z=A + 2), SHAPE), (dict(codes=A + 8), SHAPE),
    (dict(scales=A + 2), SHAPE), (dict(y=A + 4), SHAPE), (dict(n=0, z=None, codes=None, scales=None, y=None), OK)])
def test_wb_refusals(mla, over, status):
    d = {**WB, **over}
    assert mla.LIB.mla_shared_wb_mx4(d["n"], d["d_in"], d["d_out"], _p(d["z"]), _p(d["codes"]), _p(d["scales"]), d["out"],
                                     _p(d["y"]), None) == status


def test_quantize_columns_past_32_bits(mla):
    for cols, status in ((2 ** 30 + 32, UNSUPPORTED), (2 ** 31 - 32, UNSUPPORTED)):
        assert mla.LIB.mla_mx4_quantize(1, cols, _p(A), 2 ** 31, _p(A), _p(A), None) == status
        assert mla.LIB.mla_mx4_dequantize(1, cols, _p(A), _p(A), _p(A), 2 ** 31, None) == status


def test_decode_step_refusals(mla):
    """What a step could not run is refused where it is made."""
    import mx4_reference as R
    from paper_2609_07008_amd.step import DecodeStep
    for bad in (dict(n_seqs=513, n_q=2), dict(page_rows=63), dict(n_q=0), dict(n_seqs=-1), dict(geom=R.geom(64, d_c=64, d_r=16)),
                dict(geom=R.geom(129)), dict(geom=R.geom(16, n_proj_groups=3))):
        a = {**dict(geom=R.geom(16), n_seqs=2, n_q=1, max_pages=3, page_rows=64, d_out=64), **bad}
        with pytest.raises(mla.MlaError):
            DecodeStep(**a, device="cpu")


def test_stream_of_another_device(mla, monkeypatch):
    """A stream that is not of the current device is refused before anything is enqueued."""
    from types import SimpleNamespace
    other = SimpleNamespace(device_index=1, cuda_stream=0)
    with pytest.raises(mla.MlaError):
        mla._queue(other, 0)
    assert mla._queue(SimpleNamespace(device_index=0, cuda_stream=7), 0) == 7


def test_wb_channels_past_the_grid(mla):
    assert mla.LIB.mla_shared_wb_mx4(1, 64, 2 ** 24 + 1, _p(A), _p(A), _p(A), 1, _p(A), None) == UNSUPPORTED


ROWS = dict(g={}, n=2, kv=A, stride=576, slots=A, pages=4, page_rows=64, cache=A)


@pytest.mark.parametrize("over,status", [
    (dict(g=None), NULL), (dict(g=dict(d_c=64, d_r=16)), UNSUPPORTED), (dict(g=dict(value_rope=True)), UNSUPPORTED),
    (dict(g=dict(rope_base=0.5)), SHAPE), (dict(n=-1), SHAPE), (dict(stride=568), SHAPE), (dict(stride=580), SHAPE),
    (dict(page_rows=0), SHAPE), (dict(page_rows=63), SHAPE), (dict(page_rows=-64), SHAPE), (dict(page_rows=65600), UNSUPPORTED),
    (dict(pages=0), SHAPE), (dict(pages=2 ** 26), UNSUPPORTED), (dict(kv=None), NULL), (dict(slots=None), NULL), (dict(cache=None), NULL),
    (dict(kv=A + 8), SHAPE), (dict(cache=A + 8), SHAPE), (dict(slots=A + 2), SHAPE), (dict(n=2 ** 60), SHAPE),
    (dict(n=0, kv=None, slots=None, cache=None), OK)])
def test_append_and_gather_refusals(mla, over, status):
    d = {**ROWS, **over}
    g = None if d["g"] is None else ctypes.byref(mla.make_geom(R.geom(8, **d["g"])))
    assert mla.LIB.mla_cache_append(g, d["n"], _p(d["kv"]), d["stride"], None, _p(d["slots"]), d["pages"], d["page_rows"],
                                    _p(d["cache"]), None) == status
    assert mla.LIB.mla_cache_gather(g, d["n"], _p(d["slots"]), d["pages"], d["page_rows"], _p(d["cache"]), _p(d["kv"]), d["stride"],
                                    None) == status


def test_append_refuses_unaligned_positions(mla):
    g = ctypes.byref(mla.make_geom(R.geom(8)))
    assert mla.LIB.mla_cache_append(g, 2, _p(A), 576, _p(A + 2), _p(A), 4, 64, _p(A), None) == SHAPE


ATT = dict(g={}, heads=8, b=2, nq=1, q=A, pos=A, pages=A, count=A, most=3, cache_pages=4, page_rows=64, cache=A, out=A, lse=A, ws=A,
           ws_bytes=1 << 40)


@pytest.mark.parametrize("over,status", [
    (dict(g=None), NULL), (dict(g=dict(d_c=64, d_r=16)), UNSUPPORTED), (dict(g=dict(value_rope=True)), UNSUPPORTED),
    (dict(g=dict(softmax_scale=0.0)), SHAPE), (dict(b=-1), SHAPE), (dict(b=65536), UNSUPPORTED), (dict(nq=0), SHAPE),
    (dict(nq=2049), UNSUPPORTED), (dict(nq=2 ** 31 - 1), UNSUPPORTED), (dict(most=-1), SHAPE), (dict(b=60000, most=2 ** 30), UNSUPPORTED),
    (dict(page_rows=32), SHAPE), (dict(cache_pages=0), SHAPE), (dict(cache_pages=2 ** 40), UNSUPPORTED), (dict(q=None), NULL),
    (dict(pos=None), NULL), (dict(pages=None), NULL), (dict(count=None), NULL), (dict(cache=None), NULL), (dict(out=None), NULL),
    (dict(ws=None), NULL), (dict(q=A + 8), SHAPE), (dict(pages=A + 8), SHAPE), (dict(cache=A + 8), SHAPE), (dict(out=A + 8), SHAPE),
    (dict(pos=A + 1), SHAPE), (dict(count=A + 2), SHAPE), (dict(lse=A + 2), SHAPE), (dict(ws=A + 16), SHAPE),
    (dict(ws_bytes=1000), WORKSPACE), (dict(b=0, q=None, pos=None, pages=None, count=None, cache=None, out=None, ws=None, ws_bytes=0), OK)])
def test_attend_refusals(mla, over, status):
    d = {**ATT, **over}
    g = None if d["g"] is None else ctypes.byref(mla.make_geom(R.geom(d["heads"], **d["g"])))
    assert mla.LIB.mla_cache_attend(g, d["b"], d["nq"], _p(d["q"]), _p(d["pos"]), _p(d["pages"]), _p(d["count"]), d["most"],
                                    d["cache_pages"], d["page_rows"], _p(d["cache"]), _p(d["out"]), _p(d["lse"]), _p(d["ws"]),
                                    d["ws_bytes"], None) == status


def test_attend_query(mla):
    g = R.geom(64)
    small = mla.cache_attend_query(g, 1, 1, 4, 64)
    assert small % 256 == 0 and small <= mla.cache_attend_query(g, 60000, 1, 4, 64)
    assert mla.cache_attend_query(g, 0, 1, 0, 64) > 0
    ws = ctypes.c_size_t()
    assert mla.LIB.mla_cache_attend_query(ctypes.byref(mla.make_geom(g)), 1, 1, 4, 64, None) == NULL
    assert mla.LIB.mla_cache_attend_query(ctypes.byref(mla.make_geom(g)), 1, 1, 4, 65, ctypes.byref(ws)) == SHAPE


def test_binding_refuses_host_and_wrong_tensors(mla):
    """Without a GPU: a tensor in host memory never reaches the library."""
    import torch
    x = torch.zeros((2, 64), dtype=torch.bfloat16)
    c, s = torch.zeros((2, 32), dtype=torch.uint8), torch.zeros((2, 2), dtype=torch.uint8)
    kv, slots, cache = torch.zeros((2, 576), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32), torch.zeros((1, 25600), dtype=torch.uint8)
    g = R.geom(8)
    q = torch.zeros((1, 1, 8, 576), dtype=torch.bfloat16)
    i = torch.zeros((1, 1), dtype=torch.int32)
    for call in (lambda: mla.mx4_quantize(x, c, s), lambda: mla.mx4_dequantize(c, s, x),
                 lambda: mla.shared_wb_mx4(x, c, s, torch.zeros((2, 2))), lambda: mla.cache_append(g, kv, slots, cache, 64),
                 lambda: mla.cache_gather(g, slots, cache, 64, kv),
                 lambda: mla.cache_attend(g, q, i, torch.zeros((1, 2, 4), dtype=torch.int32), i[0], cache, 64,
                                          torch.zeros((1, 1, 8, 512), dtype=torch.bfloat16), workspace=cache),
                 lambda: mla.mx4_quantize(x.float(), c, s), lambda: mla.mx4_quantize(None, c, s)):
        with pytest.raises(mla.MlaError):
            call()
