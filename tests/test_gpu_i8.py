"""GPU tests of 8-bit rows (mla_i8_quantize, mla_i8_dequantize) and of W_b in them (mla_shared_wb_i8).  Codes are exact; a scale is
a quotient rounded once.  Sums of codes are exact: y takes a rounding to f32 and two products, 3 * 2^-24, and bf16 half a step, 2^-8."""
import numpy as np
import pytest

import moe_reference as R

pytestmark = pytest.mark.gpu


def _bf16_dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to(torch.bfloat16)


def _host(t):
    return t.float().cpu().numpy().astype(np.float64)


def _quantize(x):
    import torch
    from paper_2609_07008_amd import mla
    q = torch.full(x.shape, 0x5A, dtype=torch.int8, device="cuda")
    s = torch.full(x.shape[:1], -3.0, device="cuda")
    mla.i8_quantize(x, q, s)
    torch.cuda.synchronize()
    return q, s


def _same_rows(x, q, s):
    rq, rs = R.quantize(_host(x))
    assert np.array_equal(q.cpu().numpy(), rq)
    assert np.array_equal(s.cpu().numpy(), rs.astype(np.float32), equal_nan=True)


@pytest.mark.parametrize("n,c", [(1, 16), (5, 48), (3, 512), (7, 528), (2, 2048), (9, 2064), (3, 4096), (5, 4112), (2, 8192), (3, 8208), (1, 16384), (4099, 64), (0, 64)])
def test_quantize(n, c):
    rng = np.random.default_rng(n * 77 + c)
    x = _bf16_dev(rng.standard_normal((n, c)) * 2.0 ** rng.integers(-20, 20, (n, 1)))
    _same_rows(x, *_quantize(x))


def test_every_quotient_of_two_mantissas():
    """Each 8-bit mantissa over each other one at all exponents where the code is not 0: every tie, every neighbour of one."""
    m = np.arange(128, 256, dtype=np.float64)
    rows = np.concatenate([np.outer(np.ones(128), m * 2.0 ** -p) * (-1.0) ** p for p in range(10)], axis=1)    # [128, 1280]
    rows = np.where(np.abs(rows) <= m[:, None], rows, 0.0)
    rows = np.concatenate([m[:, None], rows, np.zeros((128, 15))], axis=1)
    for e in (-133, -126, -110, -108, -107, -100, -20, 0, 60, 118, 119, 120):
        x = _bf16_dev(np.ldexp(rows, e))
        _same_rows(x, *_quantize(x))


def test_odd_rows():
    x = np.ones((9, 32))
    x[0, 3], x[1, 31], x[2, 0] = np.nan, np.inf, -np.inf
    x[3] = 0.0
    x[4] = -0.0
    x[5] = 3.3895313892515355e38
    x[6] = 9.183549615799121e-41
    x[7, 0] = 3.3895313892515355e38
    x[8] = 0.0
    x[8, 17] = -1e-39
    x = _bf16_dev(x)
    _same_rows(x, *_quantize(x))


def test_strided_rows_and_back():
    import torch
    from paper_2609_07008_amd import mla
    rng = np.random.default_rng(5)
    for c, stride in ((64, 72), (4096, 4104), (528, 1024)):
        wide = _bf16_dev(rng.standard_normal((37, stride)))
        x = wide[:, :c]
        q, s = _quantize(x)
        _same_rows(x, q, s)
        back = torch.full((37, stride), 7.0, dtype=torch.bfloat16, device="cuda")
        mla.i8_dequantize(q, s, back[:, :c])
        want = q.float() * s[:, None]
        assert torch.equal(back[:, :c], want.to(torch.bfloat16)) and bool((back[:, c:] == 7).all())
    q = torch.arange(-128, 128, dtype=torch.int8, device="cuda").reshape(1, 256).repeat(2, 1)
    s = torch.tensor([0.37, float("nan")], device="cuda")
    back = torch.zeros((2, 256), dtype=torch.bfloat16, device="cuda")
    mla.i8_dequantize(q, s, back)
    assert torch.equal(back[0], (q[0].float() * s[0]).to(torch.bfloat16)) and bool(back[1].isnan().all())


def _wb(zq, zs, wq, ws, out):
    import torch
    from paper_2609_07008_amd import mla
    y = torch.full((zq.shape[0], wq.shape[0]), float("nan"), dtype=torch.bfloat16 if out == "bf16" else torch.float32, device="cuda")
    mla.shared_wb_i8(zq, zs, wq, ws, y)
    torch.cuda.synchronize()
    return y


def _inputs(n, d_in, d_out, seed):
    import torch
    gen = torch.Generator().manual_seed(seed)
    zq = torch.randint(-127, 128, (n, d_in), generator=gen, dtype=torch.int8)
    wq = torch.randint(-127, 128, (d_out, d_in), generator=gen, dtype=torch.int8)
    zs = torch.exp2(torch.randn((n,), generator=gen)) / 100
    ws = torch.exp2(torch.randn((d_out,), generator=gen)) / 100
    return zq.cuda(), zs.cuda(), wq.cuda(), ws.cuda()


def check_wb(n, d_in, d_out, out):
    import torch
    zq, zs, wq, ws = _inputs(n, d_in, d_out, n + d_in + d_out)
    y = _wb(zq, zs, wq, ws, out)
    # products of codes in float64 are whole numbers below 2^53: exact
    want = ((zq.double() @ wq.double().t()) * ws.double() * zs.double()[:, None]).cpu().numpy()
    bound = np.abs(want) * (3 * 2.0 ** -24 * (1 + 2.0 ** -7) + (2.0 ** -8 if out == "bf16" else 0))
    assert (np.abs(_host(y) - want) <= bound).all()
    bits = torch.int16 if out == "bf16" else torch.int32
    for r in {0, n // 2, n - 1}:   # a row has the same bits in any call
        assert torch.equal(_wb(zq[r:r + 1].contiguous(), zs[r:r + 1].contiguous(), wq, ws, out).view(bits), y[r:r + 1].view(bits))


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("n,d_in,d_out", [(1, 64, 1), (1, 4096, 4096), (3, 128, 17), (5, 192, 203), (16, 1088, 77), (17, 1024, 130), (31, 2112, 64), (32, 16384, 33),
                                          (33, 576, 128), (64, 960, 300), (100, 7168, 520), (130, 64, 2000), (200, 4096, 260), (257, 320, 511), (300, 128, 4100),
                                          (1000, 448, 513), (2100, 192, 1030)])
def test_wb(n, d_in, d_out, out):
    check_wb(n, d_in, d_out, out)


def test_wb_extremes():
    """The largest sums (every code 127 or -128, d_in 16384), scales of 0 and NaN."""
    import torch
    zq = torch.full((3, 16384), -128, dtype=torch.int8, device="cuda")
    wq = torch.full((5, 16384), -128, dtype=torch.int8, device="cuda")
    wq[1] = 127
    zs = torch.tensor([1.0, 0.0, float("nan")], device="cuda")
    ws = torch.tensor([1.0, 2.0, 0.0, 1e-30, float("nan")], device="cuda")
    y = _wb(zq, zs, wq, ws, "f32")
    assert y[0].tolist()[:3] == [2.0 ** 28, -2.0 * 128 * 127 * 16384, 0.0] and y[1].tolist()[:4] == [0.0, -0.0, 0.0, 0.0]
    assert bool(y[2].isnan().all()) and bool(y[:, 4].isnan().all())


def test_wb_rows_past_32_bits():
    """y rows whose offset passes 2^32 elements' bytes."""
    import torch
    n, d_in, d_out = 140000, 64, 16400
    zq, zs, wq, ws = _inputs(n, d_in, d_out, 9)
    y = _wb(zq, zs, wq, ws, "bf16")
    rows = torch.tensor([0, 65535, 130943, 130945, n - 1], device="cuda")
    want = (zq[rows].double() @ wq.double().t()) * ws.double() * zs[rows].double()[:, None]
    assert bool(((y[rows].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -22)).all())
