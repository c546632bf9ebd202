"""GPU tests of a mixture-of-experts layer (step.MoeStep: the router's product, moe_route, moe_experts_i8) as a program uses it:
against the chained 64-bit definitions, captured once and replayed, on other streams, two at a time, and a device's share of
the experts."""
import numpy as np
import pytest

import moe_reference as R
from test_gpu_experts import Layer, _tokens

pytestmark = pytest.mark.gpu


def _weights(d, experts, seed, bias=True):
    import torch
    gen = torch.Generator().manual_seed(seed)
    w_r = (torch.randn((experts, d), generator=gen) / d ** 0.5 * 2).to(torch.bfloat16).cuda()
    return w_r, (torch.randn((experts,), generator=gen) * 0.1).cuda() if bias else None


def _run(st, layer, x, w_r, bias, stream=None):
    return st.run(x, w_r, layer.w_gu, layer.s_gu, layer.w_down, layer.s_down, bias=bias, stream=stream)


CASES = [(1, 256, 128, 64, 8, dict(scoring="sigmoid", n_groups=8, top_groups=3, group_best=2, scale=2.5)),
         (37, 192, 64, 16, 4, dict(scoring="softmax", renormalize=False, min_k=2, tau=0.8)),
         (150, 128, 192, 24, 6, dict(scoring="sigmoid", min_k=3, tau=0.9))]


@pytest.mark.parametrize("n,d,f,e,k,cfg", CASES)
def test_layer(n, d, f, e, k, cfg):
    import torch
    from paper_2609_07008_amd.step import MoeStep
    layer, (w_r, bias) = Layer(d, f, e, n), _weights(d, e, n + 1, cfg["scoring"] == "sigmoid")
    x = _tokens(n, d, e, k, n + 2)[0].contiguous()
    st = MoeStep(n, d, f, e, k, y_dtype=torch.float32, with_count=True, **cfg)
    y = _run(st, layer, x, w_r, bias).cpu().numpy().astype(np.float64)
    # the router's product: at most d half steps 2^-24 of the sum of magnitudes
    xs, wr = x.double(), w_r.double()
    assert bool(((st.logits.double() - xs @ wr.t()).abs() <= d * 2.0 ** -24 * (xs.abs() @ wr.abs().t())).all())
    b = None if bias is None else bias.cpu().numpy().astype(np.float64)
    kw = {"min_k": k, "tau": 2.0, **cfg}
    idx, w, fanout = R.route(st.logits.double().cpu().numpy(), k, b, **kw)
    assert np.array_equal(st.expert_idx.cpu().numpy(), idx) and np.array_equal(st.fanout.cpu().numpy(), fanout)
    assert int(st.count.sum()) == int(fanout.sum())
    want, off, mag = layer.want(x, st.expert_idx, st.expert_w, st.fanout)
    assert (np.abs(y - want) <= off).all()


def test_shares_of_a_layer():
    """The parts of two devices, added in f32, are the layer."""
    import torch
    from paper_2609_07008_amd.step import MoeStep
    layer, (w_r, bias) = Layer(128, 64, 16, 3), _weights(128, 16, 4)
    x = _tokens(60, 128, 16, 4, 5)[0].contiguous()
    whole = _run(MoeStep(60, 128, 64, 16, 4, y_dtype=torch.float32), layer, x, w_r, bias)
    total = torch.zeros_like(whole)
    for lo, hi in ((0, 5), (5, 16)):
        part = Layer(64, 64, 1, 0)
        part.w_gu, part.s_gu, part.w_down, part.s_down = (t[lo:hi].contiguous() for t in (layer.w_gu, layer.s_gu, layer.w_down, layer.s_down))
        total += _run(MoeStep(60, 128, 64, 16, 4, n_local=hi - lo, first_expert=lo, y_dtype=torch.float32), part, x, w_r, bias)
    # a row's scale: the sums' roundings (17 half steps 2^-24 of the terms' magnitudes) are far below its largest value's 2^-16
    assert bool(((total - whole).abs().amax(1) <= whole.abs().amax(1) * 2.0 ** -16).all())


def test_captured_and_replayed():
    """One capture, replayed as x changes, with eager work and poisoned outputs between."""
    import torch
    from paper_2609_07008_amd.step import MoeStep
    n, d, f, e, k = 70, 192, 128, 24, 5
    layer, (w_r, bias) = Layer(d, f, e, 1), _weights(d, e, 2)
    args = dict(scoring="sigmoid", min_k=2, tau=0.7, with_count=True)
    st, eager = MoeStep(n, d, f, e, k, **args), MoeStep(n, d, f, e, k, **args)
    xs = [_tokens(n, d, e, k, s)[0].contiguous() for s in (20, 21, 22)]
    x = xs[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _run(st, layer, x, w_r, bias)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _run(st, layer, x, w_r, bias)
    for i in (1, 2, 0, 1):
        x.copy_(xs[i])
        for t in (st.y, st.expert_w, st.logits):
            t.fill_(float("nan"))
        st.ws.fill_(0xA5)
        st.expert_idx.fill_(-7)
        graph.replay()
        want = _run(eager, layer, xs[i], w_r, bias).clone()
        torch.cuda.synchronize()
        for a, b in ((st.y, want), (st.expert_idx, eager.expert_idx), (st.expert_w, eager.expert_w), (st.fanout, eager.fanout), (st.count, eager.count)):
            assert torch.equal(a, b)


def test_two_at_once_on_streams():
    import torch
    from paper_2609_07008_amd.step import MoeStep
    d, f, e, k = 256, 128, 16, 4
    layer, (w_r, bias) = Layer(d, f, e, 5), _weights(d, e, 6)
    xs = [_tokens(n, d, e, k, n)[0].contiguous() for n in (300, 9000)]
    steps = [MoeStep(x.shape[0], d, f, e, k, min_k=1, tau=0.6) for x in xs]
    want = [_run(st, layer, x, w_r, bias).clone() for st, x in zip(steps, xs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(5):
        for st in steps:
            st.y.fill_(float("nan"))
        torch.cuda.synchronize()
        for st, x, s in zip(steps, xs, streams):
            _run(st, layer, x, w_r, bias, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(st.y, w) for st, w in zip(steps, want))


def test_route_of_fanout_ranks():
    """The ranks that mla_moe_fanout gives from router weights feed the experts as well."""
    import torch
    from paper_2609_07008_amd import mla
    n, e, k = 40, 32, 6
    p = torch.softmax(torch.randn((n, e), generator=torch.Generator().manual_seed(3)) * 2, 1).cuda()
    idx, w = torch.zeros((n, k), dtype=torch.int32, device="cuda"), torch.zeros((n, k), device="cuda")
    fan = torch.zeros((n,), dtype=torch.int32, device="cuda")
    mla.moe_fanout(p, 0.9, idx, w, fan)
    layer = Layer(128, 64, e, 8)
    layer.check(_tokens(n, 128, e, k, 9)[0].contiguous(), idx, w, fan)
