"""GPU tests of the experts in 8 bits (mla_moe_experts_i8) against the 64-bit definition; the bound of the reference, and for a
bf16 output half a step 2^-8 of it and 2^-11 of each pair's term, which is held in f16."""
import numpy as np
import pytest

import moe_reference as R

pytestmark = pytest.mark.gpu


class Layer:
    def __init__(self, d, f, e, seed, first=0):
        import torch
        gen = torch.Generator().manual_seed(seed)
        self.d, self.f, self.e, self.first = d, f, e, first
        codes = lambda *s: torch.randn(s, generator=gen).mul(32).round().clamp(-127, 127).to(torch.int8).cuda()
        scales = lambda *s: (0.02 / 32 * torch.exp2(0.3 * torch.randn(s, generator=gen))).cuda()
        self.w_gu, self.s_gu, self.w_down, self.s_down = codes(e, 2 * f, d), scales(e, 2 * f), codes(e, d, f), scales(e, d)

    def run(self, x, idx, w, fanout=None, out="f32", ws=None, y=None):
        import torch
        from paper_2609_07008_amd import mla
        dt = torch.bfloat16 if out == "bf16" else torch.float32
        if y is None:
            y = torch.full((x.shape[0], self.d), float("nan"), dtype=dt, device="cuda")
        if ws is None:
            ws = torch.full((mla.moe_experts_i8_query(x.shape[0], self.d, self.f, self.e, idx.shape[1], dt),), 0xA5, dtype=torch.uint8, device="cuda")
        mla.moe_experts_i8(x, idx, w, self.w_gu, self.s_gu, self.w_down, self.s_down, y, ws, fanout=fanout, first_expert=self.first)
        return y

    def want(self, x, idx, w, fanout=None):
        host = lambda t: t.cpu().numpy()
        return R.experts(x.float().cpu().numpy().astype(np.float64), host(idx), host(w).astype(np.float64), None if fanout is None else host(fanout),
                         host(self.w_gu), host(self.s_gu), host(self.w_down), host(self.s_down), self.first)

    def check(self, x, idx, w, fanout=None, out="f32"):
        y = self.run(x, idx, w, fanout, out).float().cpu().numpy().astype(np.float64)
        want, off, mag = self.want(x, idx, w, fanout)
        if out == "bf16":
            off = (off + mag * 2.0 ** -11) * (1 + 2.0 ** -7) + np.abs(want) * 2.0 ** -8
        assert (np.abs(y - want) <= off).all(), (np.abs(y - want) - off).max()


def _tokens(n, d, experts, k, seed, skew=0.5, stride=None):
    import torch
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((n, stride or d), generator=gen).mul(torch.exp2(torch.randn((n, 1), generator=gen))).to(torch.bfloat16).cuda()[:, :d]
    score = torch.randn((n, experts), generator=gen) + skew * torch.randn((1, experts), generator=gen)
    idx = score.topk(k, dim=1).indices.to(torch.int32).cuda()
    w = torch.rand((n, k), generator=gen).cuda()
    fanout = torch.randint(0, k + 2, (n,), generator=gen, dtype=torch.int32).cuda()
    return x, idx, w, fanout


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,f,e,k", [(1, 64, 64, 1, 1), (1, 512, 192, 8, 2), (3, 192, 64, 4, 3), (7, 128, 320, 64, 6), (17, 320, 128, 4, 2), (33, 64, 192, 2, 1),
                                       (64, 256, 256, 16, 6), (97, 576, 64, 3, 3), (200, 128, 128, 2, 2), (300, 64, 448, 4, 2), (130, 1088, 64, 300, 8)])
def test_random(n, d, f, e, k, out):
    x, idx, w, fanout = _tokens(n, d, e, k, n + d + f)
    layer = Layer(d, f, e, e)
    layer.check(x, idx, w, None, out)
    layer.check(x, idx, w, fanout, out)


def test_widest():
    """d_model and d_ffn of 16384: the largest sums."""
    x, idx, w, _ = _tokens(2, 16384, 2, 1, 3)
    Layer(16384, 64, 2, 1).check(x, idx, w)
    x, idx, w, _ = _tokens(2, 64, 2, 2, 4)
    Layer(64, 16384, 2, 2).check(x, idx, w)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,f,k", [(1, 64, 64, 16), (2, 4160, 128, 8), (4, 192, 4160, 4), (1, 8256, 64, 3), (16, 64, 8256, 1), (3, 16384, 64, 5), (5, 128, 1088, 3),
                                     (1, 4096, 64, 1), (8, 8192, 64, 2)])
def test_few_pairs(n, d, f, k, out):
    """Up to 16 pairs, where the products find and quantize their rows themselves: all widths of their panels, all pairs at one
    expert (more than a block of rows), at different ones, some elsewhere; the bits of a call with one row more that is padding."""
    import torch
    x, idx, w, fanout = _tokens(n, d, 16, k, d + f)
    layer = Layer(d, f, 3, n + k, first=2)
    idx = idx % 6
    for i, fan in ((idx, None), (torch.full_like(idx, 3), None), (idx, fanout)):
        layer.check(x, i, w, fan, out)
        pad = 20 // k
        more = lambda t, v: None if t is None else torch.cat((t, torch.full((pad, *t.shape[1:]), v, dtype=t.dtype, device="cuda")))
        assert torch.equal(layer.run(more(x, 1), more(i, -1), more(w, 0), more(fan, 1), out)[:n], layer.run(x, i, w, fan, out))


def test_few_pairs_odd_rows():
    import torch
    x, idx, w, _ = _tokens(4, 256, 6, 3, 30)
    x[0, 9], x[1] = float("nan"), 0.0
    layer = Layer(256, 128, 6, 31)
    y = layer.run(x, idx, w)
    assert bool(y[0].isnan().all()) and bool((y[1] == 0).all()) and bool(y[2:].isfinite().all())
    assert bool((layer.run(x, torch.full_like(idx, -1), w) == 0).all())


def test_share_and_padding():
    """Experts [5, 8) of 16; indexes outside the layer; every value of fanout."""
    import torch
    x, idx, w, fanout = _tokens(90, 192, 16, 5, 8, stride=200)
    idx[80:85] = -1
    idx[85, 2], idx[86, 0], idx[87, 1] = 2 ** 31 - 1, -2 ** 31, 16
    fanout[:4] = torch.tensor([-5, 0, 100, 2 ** 31 - 1], dtype=torch.int32)
    layer = Layer(192, 128, 3, 7, first=5)
    layer.check(x, idx, w, fanout)
    layer.check(x, idx, w, None)
    y = layer.run(x, idx, w)
    gone = ~((idx >= 5) & (idx < 8)).any(1)
    assert int(gone.sum()) > 5 and bool((y[gone] == 0).all())
    y = layer.run(x, torch.full_like(idx, -1), w)
    assert bool((y == 0).all())


def test_shares_add_up():
    """Two devices' shares: each pair is in one of them."""
    import torch
    x, idx, w, _ = _tokens(40, 128, 12, 4, 9)
    whole = Layer(128, 64, 12, 5)
    parts = []
    for lo, hi in ((0, 7), (7, 12)):
        p = Layer(64, 64, 1, 0, first=lo)
        p.d, p.e = 128, hi - lo
        p.w_gu, p.s_gu, p.w_down, p.s_down = (t[lo:hi].contiguous() for t in (whole.w_gu, whole.s_gu, whole.w_down, whole.s_down))
        parts.append(p.run(x, idx, w))
    y = whole.run(x, idx, w)
    # the pairs' terms are the same; adding them up takes a product and an addition each, both at most half a step 2^-24 of
    # the sum of their magnitudes (which the shares' own sums, having cancelled, do not show): 4 + 4 in the whole, as many
    # over the shares, and the addition of the shares
    terms = sum(whole.run(x, idx[:, j:j + 1].contiguous(), w[:, j:j + 1].contiguous()).abs() for j in range(4))
    assert bool(((parts[0] + parts[1] - y).abs() <= 17 * 2.0 ** -24 * terms).all())


def test_an_expert_twice_and_all_rows_at_one():
    import torch
    x, idx, w, _ = _tokens(150, 128, 8, 3, 10)
    idx[:, 1] = idx[:, 0]
    layer = Layer(128, 64, 8, 3)
    layer.check(x, idx, w)
    layer.check(x, torch.full_like(idx, 6), w, None, "bf16")


def test_rows_do_not_meet():
    """A row's bits alone, in a batch, and again; a row of NaN, zeros and infinities beside others."""
    import torch
    x, idx, w, _ = _tokens(260, 256, 8, 3, 11)
    layer = Layer(256, 128, 8, 4)
    y = layer.run(x, idx, w)
    assert torch.equal(layer.run(x, idx, w), y)
    for r in (0, 100, 259):
        assert torch.equal(layer.run(x[r:r + 1].contiguous(), idx[r:r + 1].contiguous(), w[r:r + 1].contiguous()), y[r:r + 1])
    x2 = x.clone()
    x2[5, 7], x2[6] = float("nan"), 0.0
    x2[7, 0] = float("inf")
    y2 = layer.run(x2, idx, w)
    assert bool(y2[5].isnan().all()) and bool((y2[6] == 0).all()) and bool(y2[7].isnan().all())
    rest = torch.ones(260, dtype=torch.bool)
    rest[5:8] = False
    assert torch.equal(y2[rest], y[rest])


def test_weights_and_unused_parts():
    """Weights of NaN past the fanout, zero and negative weights; the workspace's old contents do not matter."""
    import torch
    from paper_2609_07008_amd import mla
    x, idx, w, _ = _tokens(50, 128, 8, 4, 12)
    fanout = torch.full((50,), 2, dtype=torch.int32, device="cuda")
    w[:, 2:] = float("nan")
    w[:, 1] = -w[:, 1]
    w[3] = 0.0
    layer = Layer(128, 128, 8, 6)
    layer.check(x, idx, torch.nan_to_num(w), fanout)
    y = layer.run(x, idx, w, fanout)
    ws = torch.full((mla.moe_experts_i8_query(50, 128, 128, 8, 4, torch.float32),), 0xFF, dtype=torch.uint8, device="cuda")
    assert torch.equal(layer.run(x, idx, w, fanout, ws=ws), y) and bool(y.isfinite().all())


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("n", [3, 40])
def test_activations_of_any_size(n, out):
    """h of up to 1e38, whose scale is above what a factor of 4096 leaves room for, and small ones: y in the range of ordinary numbers."""
    x, idx, w, _ = _tokens(n, 128, 4, 2, 40)
    x = x * 1024
    for up, down in ((2.0 ** 126, 2.0 ** -113), (2.0 ** -60, 2.0 ** 60)):
        layer = Layer(128, 64, 4, 41)
        layer.s_gu /= 1024
        layer.s_gu[:, 64:] *= up
        layer.s_down *= down
        y = layer.run(x, idx, w, None, out)
        assert bool(y.isfinite().all())
        layer.check(x, idx, w, None, out)


def test_no_rows():
    import torch
    x, idx, w, _ = _tokens(2, 64, 2, 1, 13)
    layer = Layer(64, 64, 2, 8)
    assert layer.run(x[:0], idx[:0], w[:0]).shape == (0, 64)


def test_thousands_of_pairs():
    """Enough pairs for every way of counting and placing them: against the pairs' own rows, computed one batch of 100 at a time."""
    import torch
    n = 9001
    x, idx, w, fanout = _tokens(n, 64, 37, 4, 14, skew=2.0)
    layer = Layer(64, 64, 37, 9)
    y = layer.run(x, idx, w, fanout)
    for lo in (0, 4000, n - 100):
        part = slice(lo, lo + 100)
        assert torch.equal(layer.run(x[part].contiguous(), idx[part].contiguous(), w[part].contiguous(), fanout[part].contiguous()), y[part])
    some = torch.randperm(n, generator=torch.Generator().manual_seed(1))[:60].cuda()
    want, off, _ = layer.want(x[some], idx[some], w[some], fanout[some])
    assert (np.abs(y[some].cpu().numpy() - want) <= off).all()


def test_rows_past_a_chunk():
    """More rows than are taken at a time: each chunk's rows as by themselves."""
    import torch
    n = 65536 + 700
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((n, 64), generator=gen, device="cuda").to(torch.bfloat16)
    idx = torch.randint(0, 5, (n, 2), generator=gen, device="cuda", dtype=torch.int32)
    w, fanout = torch.rand((n, 2), generator=gen, device="cuda"), torch.randint(0, 3, (n,), generator=gen, device="cuda", dtype=torch.int32)
    layer = Layer(64, 64, 4, 10, first=1)
    for out in ("f32", "bf16"):
        y = layer.run(x, idx, w, fanout, out)
        for lo in (0, 65400, 65536, n - 100):
            part = slice(lo, lo + 100)
            rows = layer.run(x[part].contiguous(), idx[part].contiguous(), w[part].contiguous(), fanout[part].contiguous(), out)
            assert torch.equal(rows, y[part])
    some = torch.tensor([0, 65535, 65536, n - 1], device="cuda")
    want, off, _ = layer.want(x[some], idx[some], w[some], fanout[some])
    assert (np.abs(layer.run(x, idx, w, fanout)[some].cpu().numpy() - want) <= off).all()


def test_tiles_of_every_filling():
    """Experts whose pairs fill a tile by one row, by a part of it, whole, and by a row more, in each tile height (64, 128, 256 rows
    by the pairs of an expert on average): rows as by themselves, and some against the definition."""
    import torch
    gen = torch.Generator().manual_seed(6)
    for sizes in ((1, 31, 32, 33, 63, 64, 65, 0, 130), (1, 64, 65, 127, 128, 129, 200, 0, 300, 600), (1, 33, 64, 65, 128, 129, 224, 255, 256, 257, 0, 511, 900, 1900)):
        n, e = sum(sizes), len(sizes)
        layer = Layer(320, 192, e, n)
        x = torch.randn((n, 320), generator=gen).to(torch.bfloat16).cuda()
        idx = torch.repeat_interleave(torch.arange(e), torch.tensor(sizes))[torch.randperm(n, generator=gen)].to(torch.int32).reshape(n, 1).cuda()
        w = torch.rand((n, 1), generator=gen).cuda()
        for out in ("f32", "bf16"):
            y = layer.run(x, idx, w, out=out)
            for lo in range(0, n, 150):   # other rows beside them, other tiles
                part = slice(lo, lo + 150)
                assert torch.equal(layer.run(x[part].contiguous(), idx[part].contiguous(), w[part].contiguous(), out=out), y[part])
        some = torch.randperm(n, generator=gen)[:40].cuda()
        want, off, _ = layer.want(x[some], idx[some], w[some])
        assert (np.abs(layer.run(x, idx, w)[some].cpu().numpy() - want) <= off).all()
