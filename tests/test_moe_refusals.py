"""What the router, the 8-bit calls and the experts refuse, on the host before any device work (CPU): the C ABI's checks with
made-up addresses, and the binding's checks of tensors."""
import ctypes

import pytest

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 6
A = 4096   # an aligned address that is never read
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def mla():
    from paper_2609_07008_amd import mla as m
    return m


def _p(v):
    return None if v is None else ctypes.c_void_p(v)


ROUTE = dict(n=2, e=256, logits=A, dtype=1, stride=256, bias=A, scoring=1, groups=8, kept=4, best=2, k=8, min_k=3, renorm=1, scale=1.0, tau=0.9,
             idx=A, w=A, fan=A, count=A)


@pytest.mark.parametrize("over,status", [
    (dict(n=-1), SHAPE), (dict(e=0), SHAPE), (dict(e=7, groups=1, kept=1), SHAPE), (dict(e=1025, groups=1, kept=1), UNSUPPORTED), (dict(dtype=2), SHAPE),
    (dict(scoring=2), SHAPE), (dict(scoring=-1), SHAPE), (dict(groups=0), SHAPE), (dict(groups=7), SHAPE), (dict(groups=-8), SHAPE),
    (dict(groups=128), UNSUPPORTED), (dict(kept=0), SHAPE), (dict(kept=9), SHAPE), (dict(groups=64, kept=1), SHAPE), (dict(best=0), SHAPE), (dict(best=3), SHAPE),
    (dict(k=0), UNSUPPORTED), (dict(k=9), UNSUPPORTED), (dict(min_k=0), SHAPE), (dict(min_k=9), SHAPE), (dict(scale=NAN), SHAPE), (dict(scale=INF), SHAPE),
    (dict(tau=NAN), SHAPE), (dict(stride=255), SHAPE), (dict(n=2 ** 31), UNSUPPORTED), (dict(n=2 ** 60), UNSUPPORTED), (dict(stride=2 ** 62), SHAPE), (dict(logits=None), NULL), (dict(idx=None), NULL), (dict(w=None), NULL),
    (dict(logits=A + 2), SHAPE), (dict(dtype=0, logits=A + 1), SHAPE), (dict(bias=A + 2), SHAPE), (dict(idx=A + 2), SHAPE), (dict(w=A + 1), SHAPE),
    (dict(fan=A + 2), SHAPE), (dict(count=A + 2), SHAPE), (dict(cfg=None), NULL),
    (dict(n=0, logits=None, bias=None, idx=None, w=None, fan=None, count=None), OK)])
def test_route_refusals(mla, over, status):
    d = {**ROUTE, **over}
    cfg = mla.RouteCfg(d["scoring"], d["groups"], d["kept"], d["best"], d["k"], d["min_k"], d["renorm"], d["scale"], d["tau"])
    assert mla.LIB.mla_moe_route(d["n"], d["e"], _p(d["logits"]), d["dtype"], d["stride"], _p(d["bias"]), None if "cfg" in d else ctypes.byref(cfg),
                                 _p(d["idx"]), _p(d["w"]), _p(d["fan"]), _p(d["count"]), None) == status
    assert (mla.LIB.mla_last_error_detail() == b"") == (status == OK)


QUANT = dict(n=2, c=64, x=A, stride=64, codes=A, scales=A)


@pytest.mark.parametrize("over,status", [
    (dict(n=-1), SHAPE), (dict(c=0), SHAPE), (dict(c=24), SHAPE), (dict(c=16400, stride=16400), UNSUPPORTED), (dict(stride=56), SHAPE), (dict(stride=68), SHAPE),
    (dict(x=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(x=A + 8), SHAPE), (dict(codes=A + 8), SHAPE), (dict(scales=A + 2), SHAPE),
    (dict(n=2 ** 62), SHAPE), (dict(n=0, x=None, codes=None, scales=None), OK)])
def test_quantize_refusals(mla, over, status):
    d = {**QUANT, **over}
    assert mla.LIB.mla_i8_quantize(d["n"], d["c"], _p(d["x"]), d["stride"], _p(d["codes"]), _p(d["scales"]), None) == status
    assert mla.LIB.mla_i8_dequantize(d["n"], d["c"], _p(d["codes"]), _p(d["scales"]), _p(d["x"]), d["stride"], None) == status
    assert (mla.LIB.mla_last_error_detail() == b"") == (status == OK)


WB = dict(n=2, d_in=128, d_out=8, z=A, zs=A, w=A, ws=A, out=1, y=A)


@pytest.mark.parametrize("over,status", [
    (dict(n=-1), SHAPE), (dict(d_in=0), SHAPE), (dict(d_in=96), SHAPE), (dict(d_in=16448), UNSUPPORTED), (dict(d_out=0), SHAPE),
    (dict(d_out=2 ** 24 + 1), UNSUPPORTED), (dict(n=2 ** 40), UNSUPPORTED), (dict(n=2 ** 27 + 1), UNSUPPORTED), (dict(n=2 ** 20, d_out=2 ** 20), UNSUPPORTED), (dict(out=2), SHAPE),
    (dict(z=None), NULL), (dict(zs=None), NULL), (dict(w=None), NULL), (dict(ws=None), NULL), (dict(y=None), NULL), (dict(z=A + 8), SHAPE),
    (dict(w=A + 4), SHAPE), (dict(y=A + 8), SHAPE), (dict(zs=A + 2), SHAPE), (dict(ws=A + 1), SHAPE),
    (dict(n=0, z=None, zs=None, w=None, ws=None, y=None), OK)])
def test_wb_refusals(mla, over, status):
    d = {**WB, **over}
    assert mla.LIB.mla_shared_wb_i8(d["n"], d["d_in"], d["d_out"], _p(d["z"]), _p(d["zs"]), _p(d["w"]), _p(d["ws"]), d["out"], _p(d["y"]), None) == status


EXPERTS = dict(d=128, f=64, e=4, first=0, k=2, n=3, x=A, stride=128, idx=A, w=A, fan=A, wgu=A, sgu=A, wd=A, sd=A, out=0, y=A, ws=A, ws_bytes=1 << 40)
NOTHING = dict(x=None, idx=None, w=None, fan=None, wgu=None, sgu=None, wd=None, sd=None, y=None, ws=None, ws_bytes=0)


@pytest.mark.parametrize("over,status", [
    (dict(layer=None), NULL), (dict(d=0), SHAPE), (dict(d=96), SHAPE), (dict(f=0), SHAPE), (dict(f=32), SHAPE), (dict(d=16448, stride=16448), UNSUPPORTED),
    (dict(f=16448), UNSUPPORTED), (dict(e=0), SHAPE), (dict(e=1025), UNSUPPORTED), (dict(first=-1), SHAPE), (dict(first=2 ** 31 - 3), SHAPE), (dict(k=0), SHAPE),
    (dict(k=17), UNSUPPORTED), (dict(n=-1), SHAPE), (dict(n=2 ** 62), SHAPE), (dict(out=3), SHAPE), (dict(stride=120), SHAPE),
    (dict(stride=132), SHAPE), (dict(stride=2 ** 62), SHAPE), (dict(x=None), NULL), (dict(idx=None), NULL), (dict(w=None), NULL), (dict(wgu=None), NULL),
    (dict(sgu=None), NULL), (dict(wd=None), NULL), (dict(sd=None), NULL), (dict(y=None), NULL), (dict(ws=None), NULL), (dict(x=A + 8), SHAPE), (dict(idx=A + 2), SHAPE),
    (dict(w=A + 2), SHAPE), (dict(fan=A + 2), SHAPE), (dict(wgu=A + 8), SHAPE), (dict(sgu=A + 8), SHAPE), (dict(wd=A + 8), SHAPE), (dict(sd=A + 4), SHAPE),
    (dict(y=A + 8), SHAPE), (dict(ws=A + 128), SHAPE), (dict(ws_bytes=1000), WORKSPACE), (dict(n=0, **NOTHING), OK)])
def test_experts_refusals(mla, over, status):
    d = {**EXPERTS, **over}
    layer = mla.MoeLayer(d["d"], d["f"], d["e"], d["first"], d["k"])
    assert mla.LIB.mla_moe_experts_i8(None if "layer" in d else ctypes.byref(layer), d["n"], _p(d["x"]), d["stride"], _p(d["idx"]), _p(d["w"]), _p(d["fan"]),
                                      _p(d["wgu"]), _p(d["sgu"]), _p(d["wd"]), _p(d["sd"]), d["out"], _p(d["y"]), _p(d["ws"]), d["ws_bytes"], None) == status


def test_experts_query(mla):
    import torch
    small = mla.moe_experts_i8_query(1, 4096, 2048, 256, 8)
    assert small % 256 == 0 and small < mla.moe_experts_i8_query(64, 4096, 2048, 256, 8, torch.float32)
    assert mla.moe_experts_i8_query(0, 64, 64, 1, 1) > 0
    most = mla.moe_experts_i8_query(65536, 16384, 16384, 1024, 16, torch.float32)
    assert most > 2 ** 36 and mla.moe_experts_i8_query(2 ** 40, 16384, 16384, 1024, 16, torch.float32) == most
    layer = mla.MoeLayer(64, 64, 1, 0, 1)
    assert mla.LIB.mla_moe_experts_i8_query(ctypes.byref(layer), 1, 0, None) == NULL
    with pytest.raises(mla.MlaError):
        mla.moe_experts_i8_query(1, 64, 64, 1, 1, torch.float16)


def test_binding_refuses_host_and_wrong_tensors(mla):
    """Without a GPU: a tensor in host memory never reaches the library."""
    import torch
    x, c, s = torch.zeros((2, 64), dtype=torch.bfloat16), torch.zeros((2, 64), dtype=torch.int8), torch.zeros(2)
    i, w = torch.zeros((2, 2), dtype=torch.int32), torch.zeros((2, 2))
    wgu, wd = torch.zeros((1, 128, 64), dtype=torch.int8), torch.zeros((1, 64, 64), dtype=torch.int8)
    ws = torch.zeros(4096, dtype=torch.uint8)
    for call in (lambda: mla.moe_route(torch.zeros((2, 8)), i, w), lambda: mla.moe_route(None, i, w), lambda: mla.moe_route(x.half(), i, w),
                 lambda: mla.i8_quantize(x, c, s), lambda: mla.i8_quantize(x.float(), c, s), lambda: mla.i8_dequantize(c, s, x),
                 lambda: mla.shared_wb_i8(c, s, c, s, torch.zeros((2, 2))),
                 lambda: mla.moe_experts_i8(x, i, w, wgu, torch.zeros((1, 128)), wd, torch.zeros((1, 64)), x, ws)):
        with pytest.raises(mla.MlaError):
            call()


def test_moe_step_refusals(mla):
    """What a step could not run is refused where it is made."""
    from paper_2609_07008_amd.step import MoeStep
    ok = dict(n_rows=2, d_model=128, d_ffn=64, n_experts=16, top_k=4, device="cpu")
    MoeStep(**ok)
    for bad in (dict(n_rows=-1), dict(d_model=96), dict(d_model=16448), dict(d_ffn=32), dict(n_experts=3), dict(top_k=9), dict(n_local=17), dict(n_local=0),
                dict(first_expert=1), dict(first_expert=-1, n_local=3), dict(min_k=5), dict(min_k=0), dict(tau=NAN), dict(scoring="tanh"),
                dict(n_groups=5, top_groups=5), dict(n_groups=4, top_groups=5), dict(n_groups=8, top_groups=1), dict(scale=INF)):
        with pytest.raises(mla.MlaError):
            MoeStep(**{**ok, **bad})
