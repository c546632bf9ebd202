"""W_b in 8 bits as a layer has it: rows of bf16 z quantized (mla_i8_quantize), multiplied by quantized rows of W_b (mla_shared_wb_i8),
against 64 bits, eager and captured once and replayed with new z."""
import numpy as np
import pytest

import moe_reference as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,d_in,d_out,out", [(1, 1024, 300, "f32"), (20, 576, 130, "bf16"), (200, 1984, 520, "bf16"), (700, 320, 260, "f32")])
def test_quantize_and_multiply(n, d_in, d_out, out):
    import torch
    from paper_2609_07008_amd import mla
    gen = torch.Generator().manual_seed(n)
    dt = torch.bfloat16 if out == "bf16" else torch.float32
    w = (torch.randn((d_out, d_in), generator=gen) / d_in ** 0.5).to(torch.bfloat16)
    zs = [(torch.randn((n, d_in + 8), generator=gen) * torch.exp2(torch.randn((n, 1), generator=gen))).to(torch.bfloat16) for _ in range(3)]
    z = zs[0].cuda()
    empty = lambda *s, t=torch.float32: torch.empty(s, dtype=t, device="cuda")
    wq, ws, zq, sc, y = empty(d_out, d_in, t=torch.int8), empty(d_out), empty(n, d_in, t=torch.int8), empty(n), empty(n, d_out, t=dt)
    mla.i8_quantize(w.cuda(), wq, ws)
    rw, rs = R.quantize(w.double().numpy())

    def step():
        mla.i8_quantize(z[:, :d_in], zq, sc)
        mla.shared_wb_i8(zq, sc, wq, ws, y)

    def check(i):
        q, s = R.quantize(zs[i][:, :d_in].double().numpy())
        want = (q @ rw.T) * rs * s[:, None]
        # both scales are quotients rounded once, the product takes 3 roundings, a bf16 y half a step
        bound = np.abs(want) * (5 * 2.0 ** -24 * (1 + 2.0 ** -7) + (2.0 ** -8 if out == "bf16" else 0))
        assert (np.abs(y.double().cpu().numpy() - want) <= bound).all()

    step()
    check(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (1, 2, 0, 1):
        z.copy_(zs[i])
        y.fill_(float("nan"))
        sc.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        check(i)
