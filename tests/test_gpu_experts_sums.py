"""GPU tests that the experts (mla_moe_experts_i8) hold their sums in 32 bits whatever the type of y: a bf16 y is the f32 y rounded
once, in the products of few pairs, in tiles of each height, and in a captured call."""
import numpy as np
import pytest

from test_gpu_experts import Layer, _tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,d,f,e,k", [(1, 64, 64, 1, 1), (1, 4096, 128, 16, 8), (2, 192, 4160, 16, 8), (3, 16384, 64, 8, 5), (17, 320, 128, 4, 2), (64, 1088, 256, 16, 6),
                                       (300, 64, 448, 4, 2), (700, 576, 448, 4, 1), (900, 640, 192, 4, 4), (9001, 128, 64, 37, 4)])
def test_bf16_output_is_the_f32_one_rounded(n, d, f, e, k):
    import torch
    x, idx, w, fanout = _tokens(n, d, e, k, n + d)
    layer = Layer(d, f, e, n)
    for fan in (None, fanout):
        y, y16 = layer.run(x, idx, w, fan, "f32"), layer.run(x, idx, w, fan, "bf16")
        assert torch.equal(y16, y.to(torch.bfloat16))


@pytest.mark.parametrize("n,d,f,e,k", [(2, 512, 192, 8, 2), (40, 256, 128, 8, 4), (120, 192, 320, 2, 2)])
def test_bf16_output_against_64_bits(n, d, f, e, k):
    """The reference's bound for a computation in 32 bits, and half a step 2^-8 of y for its rounding: nothing for the pairs' terms."""
    x, idx, w, _ = _tokens(n, d, e, k, 7 * n)
    layer = Layer(d, f, e, n + 1)
    y = layer.run(x, idx, w, out="bf16").float().cpu().numpy().astype(np.float64)
    want, off, _ = layer.want(x, idx, w)
    assert (np.abs(y - want) <= off * (1 + 2.0 ** -7) + np.abs(want) * 2.0 ** -8).all()
