"""Plain 64-bit definitions of the 4-bit format, the paged latent cache and the attention
over it, for the tests: numpy on the host, one row or request at a time."""
import math
from types import SimpleNamespace

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
SIGNED = np.concatenate((LEVELS, -LEVELS))


def geom(heads, d_c=512, d_r=64, **more):
    g = dict(n_heads=heads, n_groups=1, d_latent=d_c, d_rope=d_r, d_model=256, n_proj_groups=1,
             softmax_scale=1.0 / math.sqrt(192.0), rope_base=10000.0)
    g.update(more)
    return SimpleNamespace(**g)


def bf16(x):
    """The nearest bf16 values of x, ties to even, as float64 (finite x)."""
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    b = ((b.astype(np.uint64) + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).astype(np.uint32)
    return b.view(np.float32).astype(np.float64)


def quantize(x):
    """codes [n, c] (0 .. 15) and scale bytes [n, c / 32] of bf16 values x [n, c]."""
    g = np.asarray(x, dtype=np.float64).reshape(x.shape[0], x.shape[1] // 32, 32)
    bad = ~np.isfinite(g).all(-1)
    a = np.where(np.isfinite(g), np.abs(g), 0.0).max(-1)
    e = np.frexp(np.where(a > 0, a, 1.0))[1] - 3
    e = np.clip(np.where(a >= 7 * np.ldexp(1.0, e), e + 1, e), -127, 127)
    e = np.where(a > 0, e, -127)
    v = np.where(bad[..., None], 0.0, np.ldexp(np.abs(np.where(np.isfinite(g), g, 0.0)), -e[..., None]))
    code = np.zeros(g.shape, dtype=np.int64)
    for k in range(7):
        half = (LEVELS[k] + LEVELS[k + 1]) / 2
        code = np.where((v > half) | ((v == half) & (k % 2 == 1)), k + 1, code)
    code = np.where(bad[..., None], 0, code + 8 * np.signbit(g))
    return code.reshape(x.shape), np.where(bad, 255, e + 127)


def values(codes, scales):
    """What codes [n, c] and scale bytes [n, c / 32] stand for."""
    v = SIGNED[codes].reshape(codes.shape[0], codes.shape[1] // 32, 32)
    e = scales.astype(np.int64)[..., None]
    return np.where(e == 255, np.nan, np.ldexp(v, e - 127)).reshape(codes.shape)


def pack(codes):
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def unpack(b):
    out = np.empty((b.shape[0], b.shape[1] * 2), dtype=np.int64)
    out[:, 0::2], out[:, 1::2] = b & 15, b >> 4
    return out


def turned(x, angle_pos, base=10000.0):
    """x [.., 64] with its pairs (j, j + 32) turned by angle_pos [..] positions."""
    h = x.shape[-1] // 2
    a = np.asarray(angle_pos, dtype=np.float64)[..., None] * base ** (-2.0 * np.arange(h) / x.shape[-1])
    z = (x[..., :h] + 1j * x[..., h:]) * np.exp(1j * a)
    return np.concatenate((z.real, z.imag), -1)


class Cache:
    """A host copy of a paged cache tensor [pages, page_rows * 400] uint8."""

    def __init__(self, raw, page_rows):
        self.raw, self.page_rows = raw, page_rows

    def rows(self, page):
        """latent values [page_rows, 512], RoPE keys [page_rows, 64]"""
        r, p = self.page_rows, self.raw[page]
        codes = unpack(p[: r * 256].reshape(r, 256))
        scales = p[r * 256: r * 272].reshape(r, 16)
        bits = p[r * 272:].view(np.uint16).astype(np.uint32) << 16
        return values(codes, scales), bits.view(np.float32).astype(np.float64).reshape(r, 64)


def attend(g, q, pos, pages, seq_pages, cache):
    """out [B, n_q, H, 512], lse [B, n_q, H], and a bound on each output's error that a
    kernel with 32-bit sums and bf16 weights keeps: (bound of out, bound of lse)."""
    nb, nq, heads, _ = q.shape
    out = np.zeros((nb, nq, heads, 512))
    lse = np.full((nb, nq, heads), -np.inf)
    b_out, b_lse = np.zeros_like(out), np.zeros_like(lse)
    n_cache, pr = cache.raw.shape[0], cache.page_rows
    for b in range(nb):
        for j in range(nq):
            t = int(pos[b, j])
            if t < 0:
                continue
            lat, key, frames = [], [], []
            for page, rows, req, frame in pages[b, : max(0, min(int(seq_pages[b]), pages.shape[1]))].astype(np.int64):
                if not 0 <= page < n_cache:
                    continue
                n = min(max(rows, 0), pr, max(t - req + 1, 0))
                if n:
                    l, k = cache.rows(page)
                    lat.append(l[:n])
                    key.append(k[:n])
                    frames.append(np.full(n, frame))
            if not lat:
                continue
            lat, key, frames = np.concatenate(lat), np.concatenate(key), np.concatenate(frames)
            # every key turned the other way, so that the query stays as it is
            rel = turned(key, -(t - frames), g.rope_base)
            x = (q[b, j, :, :512] @ lat.T + q[b, j, :, 512:] @ rel.T) * g.softmax_scale
            with np.errstate(invalid="ignore"):
                m = x.max(-1, keepdims=True)
                p = np.exp(x - m)
                s = p.sum(-1, keepdims=True)
                w = p / s
                out[b, j] = w @ lat
                lse[b, j] = (m + np.log(s))[:, 0]
            # A score is a sum of 576 products (and the lost part of 64): its error is at most
            # 642 half steps 2^-24 of the sum of magnitudes; the turned query, kept as two bf16
            # values, adds 2^-16 of its part and the sine's 4e-7: together below 2^-14.
            mag = (np.abs(q[b, j, :, :512]) @ np.abs(lat).T + np.abs(q[b, j, :, 512:]) @ np.abs(key).T
                   + np.abs(q[b, j, :, 512:]) @ np.abs(np.roll(key, 32, 1)).T) * g.softmax_scale
            d = 2.0 ** -14 * mag.max(-1, keepdims=True)
            # a weight is off by e^d, by half a bf16 step (2^-8) and by as much of the row sum;
            # the output is rounded to bf16
            amp = w @ np.abs(lat)
            b_out[b, j] = (2 * d + 2.0 ** -8 + 2.0 ** -16) * amp + 2.0 ** -8 * np.abs(out[b, j]) + 1e-30
            b_lse[b, j] = (d + 2.0 ** -20 * (1 + np.abs(lse[b, j][:, None])))[:, 0]
    return out, lse, b_out, b_lse
