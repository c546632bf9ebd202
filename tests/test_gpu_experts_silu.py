"""GPU test of the activation h = silu(g) u of the experts (mla_moe_experts_i8), g from -87 to 87: the bf16 h next to the 64-bit
value, but where that is within 7 steps of 2^-24 of a border.

e^-|g|: the exponent's two fused steps are off by 2^-25 each, 0.7 steps of the power; the hardware's exponential 2 steps.  A
negative g takes a product with it and 1 + e, 1 each; the quotient (one Newton step) 1.1, the product with u 1: 6.8.  g and u
themselves are two products of known numbers, and taken as rounded."""
import numpy as np
import pytest

import moe_reference as R

pytestmark = pytest.mark.gpu


def run(x0, s_g, s_u):
    """h of each x0 at each expert, [experts, x0], and g and u.  An x has x0 in column 0 alone, so that its code is 127 or -127; the
    channels of a row are alike, so that h is 127 times the row's scale, to two roundings, and has 8 bits."""
    import torch
    from paper_2609_07008_amd import mla
    e, d, f, n = len(s_g), 64, 64, len(s_g) * len(x0)
    x = torch.zeros((e, len(x0), d), dtype=torch.bfloat16, device="cuda")
    x[:, :, 0] = torch.from_numpy(x0).cuda()
    w_gu, w_down = torch.zeros((e, 2 * f, d), dtype=torch.int8, device="cuda"), torch.zeros((e, d, f), dtype=torch.int8, device="cuda")
    w_gu[:, :, 0], w_down[:, :, 0] = 127, 1
    s_gu = torch.from_numpy(np.repeat(np.stack((s_g, s_u), 1), f, 1)).cuda()
    idx = torch.arange(e, dtype=torch.int32, device="cuda").repeat_interleave(len(x0)).reshape(n, 1)
    y = torch.full((n, d), float("nan"), device="cuda")
    ws = torch.empty((mla.moe_experts_i8_query(n, d, f, e, 1, torch.float32),), dtype=torch.uint8, device="cuda")
    mla.moe_experts_i8(x.reshape(n, d), idx, torch.ones((n, 1), device="cuda"), w_gu, s_gu, w_down, torch.ones((e, d), device="cuda"), y, ws)
    assert bool((y == y[:, :1]).all())
    acc, xs = (np.sign(x0) * 127 * 127).astype(np.float32), np.abs(x0).astype(np.float32) / np.float32(127)
    g, u = (((acc * s[:, None]) * xs).astype(np.float64) for s in (s_g, s_u))
    return R.bf16(y[:, 0].cpu().numpy().astype(np.float64)).reshape(e, len(x0)), g, u


def scales(e, seed):
    rng = np.random.default_rng(seed)
    return rng.uniform(0.3, 0.68, e).astype(np.float32) / np.float32(127), rng.uniform(1.0, 2.0, e).astype(np.float32) * np.float32(2.0 ** 20)


def check(h, g, u):
    v = g / (1.0 + np.exp(-g)) * u
    # h = 127 * (w h / 127): the code of a negative h is -127
    lo, hi = R.bf16(v * (1 - 7 * 2.0 ** -24)), R.bf16(v * (1 + 7 * 2.0 ** -24))
    bad = (h != lo) & (h != hi)
    assert not bad.any(), (int(bad.sum()), bad.size, g[bad][:5], h[bad][:5], v[bad][:5])


def test_large_arguments():
    """Some 400,000 of either sign, where an exponent rounded to f32 is off by up to 44 steps."""
    x0 = np.ldexp(np.arange(128, 256, dtype=np.float64)[None, :], np.arange(-3, 0)[:, None]).ravel()   # 16 .. 128
    check(*run(np.concatenate((x0, -x0)), *scales(1024, 3)))


def test_small_arguments():
    x0 = np.ldexp(np.arange(128, 256, dtype=np.float64)[None, :], np.arange(-13, -3)[:, None]).ravel()   # 2^-6 .. 16
    check(*run(np.concatenate((x0, -x0)), *scales(100, 4)))


def test_few_pairs():
    """The products that quantize their rows themselves: 16 rows a call."""
    for seed in range(8):
        x0 = np.random.default_rng(seed).integers(128, 256, 16) * 2.0 ** (seed % 4 - 4) * np.where(np.arange(16) % 2, 1.0, -1.0)
        check(*run(x0, *scales(1, 50 + seed)))


def test_ends():
    """Arguments past the exponential's range: silu(g) is g, or nothing."""
    h, g, u = run(np.ldexp(np.array([1.0, -1.0, 1.0, -1.0, 1.0, -1.0]), [20, 20, 60, 60, 120, 120]), np.float32([1 / 127]), np.float32([2.0 ** -126]))
    v = np.where(g > 0, g, 0.0) * u
    assert (np.abs(h - v) <= np.abs(v) * (2.0 ** -8 + 2.0 ** -20)).all() and (h[g < 0] == 0).all()
