"""A padded batch through step.MoeStep: the caller marks rows with an index of -1 between routing and experts; their y is 0, the
other rows have the bits of the unpadded batch, and no expert's weights are met for them."""
import pytest

from test_gpu_experts import Layer, _tokens
from test_gpu_moe_step import _weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,real", [(64, 40), (8, 1), (300, 299)])
def test_rows_marked_as_padding(rows, real):
    import torch
    from paper_2609_07008_amd.step import MoeStep
    d, f, e, k = 192, 128, 16, 3
    layer, (w_r, bias) = Layer(d, f, e, rows), _weights(d, e, real)
    x = _tokens(rows, d, e, k, 7)[0].contiguous()
    x[real:] = float("nan")
    st, alone = MoeStep(rows, d, f, e, k, scoring="sigmoid"), MoeStep(real, d, f, e, k, scoring="sigmoid")
    args = (layer.w_gu, layer.s_gu, layer.w_down, layer.s_down)
    want = alone.run(x[:real].contiguous(), w_r, *args, bias=bias)
    st.route(x, w_r, bias)
    st.expert_idx[real:] = -1
    st.experts(x, *args)
    assert torch.equal(st.y[:real], want) and bool((st.y[real:] == 0).all())
