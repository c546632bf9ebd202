"""GPU test of experts that every row uses (mla_moe_experts_i8): columns in front of a router's, counted in the fanout, are used
whatever the row's own fanout; columns at or past the fanout are not."""
import pytest

from test_gpu_experts import Layer, _tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [2, 60])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_experts_in_front(n, out):
    import torch
    x, idx, w, _ = _tokens(n, 192, 6, 4, n)
    layer = Layer(192, 128, 8, n + 1)
    fanout = (torch.arange(n, device="cuda", dtype=torch.int32) % 4) + 1
    front = torch.tensor([6, 7], dtype=torch.int32, device="cuda").expand(n, 2)
    ones = torch.ones((n, 2), device="cuda")
    idx2, w2 = torch.cat((front, idx), 1).contiguous(), torch.cat((ones, w), 1).contiguous()
    layer.check(x, idx2, w2, fanout + 2, out)
    # what they add is there: the same rows without them differ
    assert bool((layer.run(x, idx2, w2, fanout + 2, out) != layer.run(x, idx, w, fanout, out)).any(1).all())
    # behind the router's columns they lie past the fanout and add nothing
    idx3, w3 = torch.cat((idx, front), 1).contiguous(), torch.cat((w, ones), 1).contiguous()
    assert torch.equal(layer.run(x, idx3, w3, fanout, out), layer.run(x, idx, w, fanout, out))
