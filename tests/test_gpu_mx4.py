"""GPU tests of the 4-bit format (mla_mx4_quantize, mla_mx4_dequantize) and of W_b in it
(mla_shared_wb_mx4) against plain 64-bit definitions.  Quantizing is exact, so codes and
scales are compared bit for bit.  A product's sums are in 32 bits: at most d_in half steps
2^-24 of the sum of magnitudes, and half a step of a bf16 output."""
import numpy as np
import pytest

import mx4_reference as R

pytestmark = pytest.mark.gpu


def _bf16_dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to(torch.bfloat16)


def _host(t):
    return t.float().cpu().numpy().astype(np.float64)


def _quantize(x):
    import torch
    from paper_2609_07008_amd import mla
    codes = torch.full((x.shape[0], x.shape[1] // 2), 0x5A, dtype=torch.uint8, device="cuda")
    scales = torch.full((x.shape[0], x.shape[1] // 32), 0x5A, dtype=torch.uint8, device="cuda")
    mla.mx4_quantize(x, codes, scales)
    torch.cuda.synchronize()
    return codes, scales


@pytest.mark.parametrize("n,c", [(1, 32), (3, 64), (7, 96), (5, 480), (2, 512), (9, 544), (33, 2016), (1, 16384), (0, 64)])
def test_quantize_and_back(n, c):
    import torch
    from paper_2609_07008_amd import mla
    rng = np.random.default_rng(n * 1000 + c)
    x = _bf16_dev(rng.standard_normal((n, c)) * 2.0 ** rng.integers(-20, 20, (n, 1)))
    codes, scales = _quantize(x)
    want_c, want_s = R.quantize(_host(x)) if n else (np.zeros((0, c), dtype=np.int64), np.zeros((0, c // 32)))
    assert np.array_equal(codes.cpu().numpy(), R.pack(want_c)) and np.array_equal(scales.cpu().numpy(), want_s)
    back = torch.full((n, c), 7.0, dtype=torch.bfloat16, device="cuda")
    mla.mx4_dequantize(codes, scales, back)
    torch.cuda.synchronize()
    assert np.array_equal(_host(back), R.values(want_c, want_s.astype(np.int64)))


def test_quantize_every_scale_edge():
    """Group maxima around every threshold of the scale (6.5, 7, 7.5 units), ties of every
    level, signed zeros, the smallest and largest values, NaN and infinities."""
    rows = []
    for p in (-133, -130, -127, -126, -125, -120, -3, 0, 60, 120, 125):
        for top in (4.0, 5.0, 6.0, 6.5, 6.96875, 7.0, 7.5, 7.96875):
            v = np.zeros(32)
            v[:17] = [top, .25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5.0, -0.0, .2421875]
            with np.errstate(over="ignore"):
                rows.append(np.ldexp(v, p))
    for odd in (np.nan, np.inf, -np.inf):
        v = np.ones(32)
        v[31] = odd
        rows.append(v)
    rows += [np.zeros(32), -np.zeros(32), np.full(32, 3.3895313892515355e38), np.full(32, 9.183549615799121e-41)]
    x = _bf16_dev(np.stack(rows))
    assert np.array_equal(np.isfinite(_host(x)), np.isfinite(np.stack(rows)))
    codes, scales = _quantize(x)
    want_c, want_s = R.quantize(_host(x))
    assert np.array_equal(codes.cpu().numpy(), R.pack(want_c)) and np.array_equal(scales.cpu().numpy(), want_s)


def test_dequantize_every_code_and_scale():
    import torch
    from paper_2609_07008_amd import mla
    b = np.arange(256, dtype=np.uint8)
    codes = np.tile(b.reshape(16, 16), (256, 1))                       # each scale meets every byte
    scales = np.repeat(b, 16)[:, None]
    x = torch.zeros((4096, 32), dtype=torch.bfloat16, device="cuda")
    mla.mx4_dequantize(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), x)
    torch.cuda.synchronize()
    with np.errstate(over="ignore"):
        want = R.values(R.unpack(codes), scales).astype(np.float32)    # 6 x 2^127 passes the range: infinite
    assert np.array_equal(x.float().cpu().numpy(), want, equal_nan=True)


def test_quantize_strided_rows():
    import torch
    from paper_2609_07008_amd import mla
    rng = np.random.default_rng(5)
    wide = _bf16_dev(rng.standard_normal((37, 200)))
    x = wide[:, 8:168]
    assert x.stride(0) == 200
    codes, scales = _quantize(x)
    want_c, want_s = R.quantize(_host(x))
    assert np.array_equal(codes.cpu().numpy(), R.pack(want_c)) and np.array_equal(scales.cpu().numpy(), want_s)
    back = torch.full((37, 200), 7.0, dtype=torch.bfloat16, device="cuda")
    mla.mx4_dequantize(codes, scales, back[:, 8:168])
    torch.cuda.synchronize()
    got = _host(back)
    assert np.array_equal(got[:, 8:168], R.values(want_c, want_s))
    assert (got[:, :8] == 7).all() and (got[:, 168:] == 7).all()       # beside the view: as it was


def _weight(d_out, d_in, seed):
    rng = np.random.default_rng(seed)
    w = R.bf16(rng.standard_normal((d_out, d_in)) * 0.05)
    c, s = R.quantize(w)
    return c, s


def _wb(z, c, s, out):
    import torch
    from paper_2609_07008_amd import mla
    y = torch.full((z.shape[0], c.shape[0]), float("nan"), device="cuda",
                   dtype=torch.bfloat16 if out == "bf16" else torch.float32)
    mla.shared_wb_mx4(z, torch.from_numpy(R.pack(c)).cuda(), torch.from_numpy(s.astype(np.uint8)).cuda(), y)
    torch.cuda.synchronize()
    return y


SHAPES = [(1, 64, 1), (1, 64, 3), (2, 128, 17), (16, 192, 40), (17, 448, 100), (32, 512, 65), (33, 576, 130), (64, 1024, 256),
          (65, 2048, 77), (129, 320, 500), (200, 4096, 48), (5, 16384, 33), (1, 4096, 4096), (40, 7168, 20), (1024, 64, 33)]


@pytest.mark.parametrize("n,d_in,d_out", SHAPES)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_wb_mx4(n, d_in, d_out, out):
    rng = np.random.default_rng(n + d_in + d_out)
    z = _bf16_dev(rng.standard_normal((n, d_in)))
    c, s = _weight(d_out, d_in, d_in + d_out)
    y = _wb(z, c, s, out)
    w, zz = R.values(c, s), _host(z)
    want = zz @ w.T
    bound = d_in * 2.0 ** -24 * (np.abs(zz) @ np.abs(w).T) + 1e-30
    if out == "bf16":
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    assert (np.abs(_host(y) - want) <= bound).all()


def test_wb_mx4_rows_alike_in_any_call():
    import torch
    rng = np.random.default_rng(3)
    z = _bf16_dev(rng.standard_normal((300, 1088)))
    c, s = _weight(210, 1088, 4)
    full = _wb(z, c, s, "f32")
    for lo, hi in ((0, 1), (7, 8), (0, 16), (3, 20), (100, 133), (290, 300), (40, 140)):
        assert torch.equal(_wb(z[lo:hi].contiguous(), c, s, "f32").view(torch.int32), full[lo:hi].contiguous().view(torch.int32))


# every tile, its last block of rows and of channels ragged; d_in: whole steps, a half slab, fewer slabs than a step
TILES = [(5, 200, 1088), (31, 1001, 192), (16, 6150, 320), (32, 6150, 1088), (9, 12300, 448), (30, 12300, 576), (150, 6150, 1088),
         (190, 12300, 320)]


@pytest.mark.parametrize("n,d_out,d_in", TILES)
def test_wb_mx4_tiles(n, d_out, d_in):
    """One answer from every tile: against 64 bits, and a row alone in the same bits."""
    import torch
    rng = np.random.default_rng(n + d_in + d_out)
    z = _bf16_dev(rng.standard_normal((n, d_in)))
    c, s = _weight(d_out, d_in, d_in + d_out)
    y = _wb(z, c, s, "f32")
    w, zz = R.values(c, s), _host(z)
    assert (np.abs(_host(y) - zz @ w.T) <= d_in * 2.0 ** -24 * (np.abs(zz) @ np.abs(w).T) + 1e-30).all()
    for row in (0, n // 2, n - 1):
        assert torch.equal(_wb(z[row:row + 1].contiguous(), c, s, "f32").view(torch.int32), y[row:row + 1].view(torch.int32))


def test_wb_mx4_nan_scale_and_infinite_row():
    """A NaN group reaches its channel alone, an infinite z its row alone."""
    rng = np.random.default_rng(8)
    x = rng.standard_normal((20, 192))
    x[4, 100] = np.inf
    z = _bf16_dev(x)
    c, s = _weight(50, 192, 9)
    s[13, 5] = 255
    got = _host(_wb(z, c, s, "f32"))
    bad = ~np.isfinite(got)
    want = np.zeros_like(bad)
    want[4] = True
    want[:, 13] = True
    assert np.array_equal(bad, want)


def test_wb_mx4_agrees_with_dequantized_shared_wb():
    """The same products as mla_shared_wb on the unpacked weight, in another order."""
    import torch
    from paper_2609_07008_amd import mla
    rng = np.random.default_rng(12)
    z = _bf16_dev(rng.standard_normal((24, 1024)))
    c, s = _weight(300, 1024, 13)
    w = torch.empty((300, 1024), dtype=torch.bfloat16, device="cuda")
    mla.mx4_dequantize(torch.from_numpy(R.pack(c)).cuda(), torch.from_numpy(s.astype(np.uint8)).cuda(), w)
    y = torch.empty((24, 300), dtype=torch.float32, device="cuda")
    mla.shared_wb(z, w, y)
    bound = 2 * 1024 * 2.0 ** -24 * (np.abs(_host(z)) @ np.abs(R.values(c, s)).T)
    assert (np.abs(_host(y) - _host(_wb(z, c, s, "f32"))) <= bound).all()
