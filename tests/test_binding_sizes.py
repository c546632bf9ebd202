"""The binding on the CPU: a number that the C ABI's 32-bit arguments cannot hold is refused, not cut to its lower bits.  Tensors are
of torch's meta device (shapes without memory), taken as the current one; no call gets past its checks."""
from types import SimpleNamespace

import pytest

BIG = 2 ** 32 + 64   # its lower 32 bits are a size that every call takes


@pytest.fixture
def mla(monkeypatch):
    from paper_2609_07008_amd import mla as m
    monkeypatch.setattr(m, "_device", lambda: -1)
    return m


STREAM = SimpleNamespace(device_index=-1, cuda_stream=0)


def _t(dtype, *shape):
    import torch
    return torch.empty(shape, dtype=getattr(torch, dtype), device="meta")


def _refused(mla, call):
    with pytest.raises(mla.MlaError, match=str(BIG)) as e:
        call()
    assert e.value.status == 3   # MLA_ERR_UNSUPPORTED


def test_plain_numbers(mla):
    from paper_2609_07008_amd.step import MoeStep
    ok = dict(n_experts=256, top_k=8, n_groups=8, top_groups=4, group_best=2, min_k=3)
    mla.check_route(**ok)
    for name in ok:
        _refused(mla, lambda: mla.check_route(**{**ok, name: BIG}))
    layer = dict(n_rows=5, d_model=64, d_ffn=64, n_experts=64, top_k=1)
    mla.moe_experts_i8_query(**layer)
    for name in ("d_model", "d_ffn", "n_experts", "top_k"):
        _refused(mla, lambda: mla.moe_experts_i8_query(**{**layer, name: BIG}))
    for n in (2 ** 64 + 5, -2 ** 64 + 5):
        with pytest.raises(mla.MlaError):
            mla.moe_experts_i8_query(**{**layer, "n_rows": n})
    with pytest.raises(mla.MlaError):
        MoeStep(2, 128, 64, BIG, 4, device="cpu", n_local=16, first_expert=2 ** 32)


def test_route(mla):
    _refused(mla, lambda: mla.moe_route(_t("float32", 1, BIG), _t("int32", 1, 4), _t("float32", 1, 4), stream=STREAM))
    _refused(mla, lambda: mla.moe_route(_t("float32", 1, 64), _t("int32", 1, 4), _t("float32", 1, 4), n_groups=BIG, stream=STREAM))
    _refused(mla, lambda: mla.moe_route(_t("float32", 1, 64), _t("int32", 1, BIG), _t("float32", 1, BIG), stream=STREAM))


def test_rows_in_8_and_4_bits(mla):
    _refused(mla, lambda: mla.i8_quantize(_t("bfloat16", 1, BIG), _t("int8", 1, BIG), _t("float32", 1), stream=STREAM))
    _refused(mla, lambda: mla.i8_dequantize(_t("int8", 1, BIG), _t("float32", 1), _t("bfloat16", 1, BIG), stream=STREAM))
    _refused(mla, lambda: mla.mx4_quantize(_t("bfloat16", 1, BIG), _t("uint8", 1, BIG // 2), _t("uint8", 1, BIG // 32), stream=STREAM))
    _refused(mla, lambda: mla.mx4_dequantize(_t("uint8", 1, BIG // 2), _t("uint8", 1, BIG // 32), _t("bfloat16", 1, BIG), stream=STREAM))


@pytest.mark.parametrize("d_in,d_out", [(BIG, 8), (128, BIG)])
def test_wb(mla, d_in, d_out):
    y, s = _t("float32", 1, d_out), _t("float32", d_out)
    _refused(mla, lambda: mla.shared_wb_i8(_t("int8", 1, d_in), _t("float32", 1), _t("int8", d_out, d_in), s, y, stream=STREAM))
    _refused(mla, lambda: mla.shared_wb_mx4(_t("bfloat16", 1, d_in), _t("uint8", d_out, d_in // 2), _t("uint8", d_out, d_in // 32), y, stream=STREAM))
    _refused(mla, lambda: mla.shared_wb(_t("bfloat16", 1, d_in), _t("bfloat16", d_out, d_in), y, stream=STREAM))


@pytest.mark.parametrize("over", [dict(d=BIG), dict(f=BIG), dict(e=BIG), dict(k=BIG), dict(first=BIG)])
def test_experts(mla, over):
    s = {**dict(d=64, f=64, e=64, k=2, first=0), **over}
    d, f, e, k = s["d"], s["f"], s["e"], s["k"]
    _refused(mla, lambda: mla.moe_experts_i8(_t("bfloat16", 1, d), _t("int32", 1, k), _t("float32", 1, k), _t("int8", e, 2 * f, d), _t("float32", e, 2 * f),
                                             _t("int8", e, d, f), _t("float32", e, d), _t("float32", 1, d), _t("uint8", 4096), first_expert=s["first"],
                                             stream=STREAM))
