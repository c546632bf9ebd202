"""GPU test that the experts (mla_moe_experts_i8) run in one workspace from the largest batch down to a single row, and write
nothing behind the bytes that the query names for that batch."""
import pytest

from test_gpu_experts import Layer, _tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("most,d,f,e,k", [(20, 512, 256, 8, 1), (17, 192, 64, 4, 3), (400, 128, 192, 2, 2), (900, 64, 128, 2, 1)])
def test_one_workspace_for_every_batch(most, d, f, e, k):
    import torch
    from paper_2609_07008_amd import mla
    x, idx, w, fanout = _tokens(most, d, e, k, most)
    layer = Layer(d, f, e, most)
    need = mla.moe_experts_i8_query(most, d, f, e, k, torch.bfloat16)
    room = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    for n in sorted({most, most - 1, most // 2, 17, 16, 15, 16 // k, 1, 257, 258, 259, 769, 770} & set(range(1, most + 1)), reverse=True):
        cut = lambda t: t[:n].contiguous()
        y = layer.run(cut(x), cut(idx), cut(w), cut(fanout), "bf16", ws=room[:need])
        assert torch.equal(y, layer.run(cut(x), cut(idx), cut(w), cut(fanout), "bf16"))
        assert bool((room[need:] == 0xA5).all())
