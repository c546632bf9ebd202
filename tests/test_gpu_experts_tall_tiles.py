"""The experts in 8 bits (mla_moe_experts_i8) in each tile height with several column tiles, more than one group of row tiles of an
expert, and K of more than twice the slices that a tile keeps in LDS, whole and half last ones: every filling of a tile.  Rows are
the bits of calls in lower tiles and of the few-pair products, and some are held to the 64-bit definition.  That the sizes
have these heights is asserted on the CPU, of the library's own rule (test_i8_rules.py)."""
import numpy as np
import pytest

from test_gpu_experts import Layer

pytestmark = pytest.mark.gpu

# pairs of each expert, by the height of the tiles
SIZES = {64: (1, 31, 32, 33, 63, 64, 65, 0, 130, 590), 128: (1, 64, 65, 127, 128, 129, 200, 0, 300, 1200),
         256: (1, 64, 65, 128, 129, 255, 257, 0, 700, 2400)}
WIDTHS = ((1088, 960), (1024, 832))   # d_model, d_ffn: 8.5 and 7.5 slices, 8 and 6.5
SLICES = 3                             # that a tile keeps in LDS, at most


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("d,f", WIDTHS)
@pytest.mark.parametrize("rows", list(SIZES))
def test_every_filling(rows, d, f, out):
    import torch
    sizes = SIZES[rows]
    gen = torch.Generator().manual_seed(rows + d)
    n, e = sum(sizes), len(sizes)
    layer = Layer(d, f, e, rows)
    x = torch.randn((n, d), generator=gen).to(torch.bfloat16).cuda()
    idx = torch.repeat_interleave(torch.arange(e), torch.tensor(sizes))[torch.randperm(n, generator=gen)].to(torch.int32).reshape(n, 1).cuda()
    w = torch.rand((n, 1), generator=gen).cuda()
    y = layer.run(x, idx, w, out=out)
    cut = lambda t, lo, hi: t[lo:hi].contiguous()
    for lo in range(0, n, 150):   # other rows beside them, the lowest tiles
        assert torch.equal(layer.run(cut(x, lo, lo + 150), cut(idx, lo, lo + 150), cut(w, lo, lo + 150), out=out), y[lo:lo + 150])
    for lo in range(0, n, 499):   # few pairs
        assert torch.equal(layer.run(cut(x, lo, lo + 16), cut(idx, lo, lo + 16), cut(w, lo, lo + 16), out=out), y[lo:lo + 16])
    some = torch.randperm(n, generator=gen)[:30].cuda()
    want, off, _ = layer.want(x[some], idx[some], w[some])
    got = y[some].float().cpu().numpy().astype(np.float64)
    if out == "bf16":
        off = off * (1 + 2.0 ** -7) + np.abs(want) * 2.0 ** -8
    assert (np.abs(got - want) <= off).all()


@pytest.mark.parametrize("rows", list(SIZES))
def test_several_pairs_a_row(rows):
    """top_k of 3 with a fanout: rows of different experts' tiles meet at the join."""
    import torch
    d, f = 576, 448
    sizes = SIZES[rows]
    gen = torch.Generator().manual_seed(rows)
    e = len(sizes)
    total = sum(sizes) // 3 * 3
    expert = torch.repeat_interleave(torch.arange(e), torch.tensor(sizes))[torch.randperm(sum(sizes), generator=gen)][:total]
    idx = expert.to(torch.int32).reshape(total // 3, 3).cuda()
    n = total // 3
    x, w = torch.randn((n, d), generator=gen).to(torch.bfloat16).cuda(), torch.rand((n, 3), generator=gen).cuda()
    fanout = torch.randint(0, 4, (n,), generator=gen, dtype=torch.int32).cuda()
    layer = Layer(d, f, e, rows + 1)
    for fan in (None, fanout):
        y = layer.run(x, idx, w, fan)
        for lo in range(0, n, 5):
            part = slice(lo, lo + 5)
            cut = lambda t: None if t is None else t[part].contiguous()
            if lo % 3 == 0:
                assert torch.equal(layer.run(cut(x), cut(idx), cut(w), cut(fan)), y[part])
        some = torch.randperm(n, generator=gen)[:20].cuda()
        want, off, _ = layer.want(x[some], idx[some], w[some], None if fan is None else fan[some])
        assert (np.abs(y[some].cpu().numpy() - want) <= off).all()
