"""Plain 64-bit definitions of the router, of 8-bit rows and of the experts' products, for the tests (numpy)."""
import numpy as np


def route(x, top_k, bias=None, scoring="softmax", n_groups=1, top_groups=1, group_best=1, renormalize=True, scale=1.0, min_k=1, tau=2.0):
    """(idx, w, fanout) of 64-bit logits x [N, E]; equal values go to the lower index, NaN behind every number."""
    n, e = x.shape
    with np.errstate(all="ignore"):
        if scoring == "softmax":
            m = np.where(np.isnan(x), -np.inf, x).max(1, keepdims=True)
            p = np.where((m == -np.inf) & (x == m), 0.0, np.exp(x - m))
            total = p.sum(1, keepdims=True)
            p = np.where(total == 0, p, p / total)
        else:
            p = 1.0 / (1.0 + np.exp(-x))
        c = p if bias is None else p + bias
    size = e // n_groups

    def order(v):   # descending, stable, NaN last
        return np.argsort(np.where(np.isnan(v), np.inf, -v), axis=1, kind="stable"), np.isnan(v)

    def ranked(v):
        first, nan = order(v)
        # -infinity and NaN share a key above: move NaN behind
        return np.take_along_axis(first, np.argsort(np.take_along_axis(nan, first, 1), axis=1, kind="stable"), 1)

    by = x if bias is None else c
    if top_groups < n_groups:
        g = c.reshape(n, n_groups, size)
        best = np.take_along_axis(g.reshape(n * n_groups, size), ranked(g.reshape(n * n_groups, size)), 1)[:, :min(group_best, size)]
        with np.errstate(all="ignore"):
            score = best.sum(1).reshape(n, n_groups)
        place = np.argsort(ranked(score), axis=1, kind="stable")
        open_ = np.repeat(place < top_groups, size, axis=1)
    else:
        open_ = np.ones((n, e), dtype=bool)
    full = ranked(by)
    kept = np.take_along_axis(open_, full, 1)
    idx = np.take_along_axis(full, np.argsort(~kept, axis=1, kind="stable"), 1)[:, :top_k]
    s = np.take_along_axis(p, idx, 1)
    total = s.sum(1)
    upto = np.zeros(n)
    fanout = np.full(n, top_k)
    done = np.zeros(n, dtype=bool)
    with np.errstate(all="ignore"):
        for j in range(top_k):
            upto = upto + s[:, j]
            hit = ~done & (j + 1 >= min_k) & (total > 0) & (upto >= float(np.float32(tau)) * total)
            fanout[hit] = j + 1
            done |= hit
        w = s / np.where(total == 0, 1.0, total)[:, None] if renormalize else s
        return idx.astype(np.int32), w * float(np.float32(scale)), fanout.astype(np.int32)


def quantize(x):
    """Codes (int64) and scales (64 bits) of rows of bf16 values x; the quotient of 127 x and max|x| decides exactly."""
    top = np.abs(x).max(-1, keepdims=True) if x.shape[-1] else np.zeros(x.shape[:-1] + (1,))
    bad = ~np.isfinite(x).all(-1, keepdims=True)
    safe = np.where(bad | (top == 0), 1.0, top)
    q = np.where(bad, 0.0, np.rint(np.where(bad, 0.0, x) * 127.0 / safe)).astype(np.int64)
    return q, np.where(bad, np.nan, top / 127.0)[..., 0]


def bf16(x):
    """64-bit values to the nearest bf16 (ties to even), as 64 bits."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(np.ldexp(m, 8)), np.maximum(e, -125) - 8) if np.all(np.abs(x[x != 0]) > 1e-37) else _bf16_any(x)


def _bf16_any(x):
    m, e = np.frexp(x)
    step = np.maximum(e - 8, -133)
    return np.ldexp(np.rint(np.ldexp(x, -step)), step)


def experts(x, idx, w, fanout, w_gu, s_gu, w_down, s_down, first=0):
    """(y, off, mag) [N, d]: y of the definition, how far a computation with 32-bit steps may be from it, and the sum of the
    magnitudes of its pairs' terms.  (Where the terms are held in f16 before they are summed, half a step 2^-11 of each comes on top.)

    A product's sum is exact and then takes three roundings (to f32, two scales): relative 3 * 2^-24.  Of h = silu(g) u: g's
    error counts (1 + |g|) times in silu, the exponential's is at most (1.5 |g| + 2) steps of 2^-24, and the other operations
    (the second factor's 3 roundings, 1 + e, the reciprocal's 2, two products) 8 more: (4.5 |g| + 13) * 2^-24 in all, taken as
    (5 |g| + 13).  Where a bf16 border
    is nearer than that, h may be the neighbour, a step of at most 2^-7 of it, and its code another one; where that is the row's
    largest value every code may be another one, and the scale is 2^-7 off.  The sum over the pairs takes a product and an addition
    each, and parts three roundings."""
    n, d = x.shape
    f = w_down.shape[2]
    xq, xs = quantize(x)
    y, off, mag = np.zeros((n, d)), np.zeros((n, d)), np.zeros((n, d))
    for r in range(n):
        for j in range(idx.shape[1] if fanout is None else min(idx.shape[1], int(fanout[r]))):
            e = int(idx[r, j]) - first
            if not 0 <= e < w_down.shape[0]:
                continue
            gu = (w_gu[e].astype(np.int64) @ xq[r]) * s_gu[e].astype(np.float64) * xs[r]
            g, u = gu[:f], gu[f:]
            with np.errstate(over="ignore"):
                v = g / (1.0 + np.exp(-g)) * u
            h = bf16(v)
            err = np.abs(v) * (5 * np.abs(g) + 13) * 2.0 ** -24
            odd = (bf16(v - err) != h) | (bf16(v + err) != h)
            hq, hs = quantize(h[None])
            dh = np.where(odd, np.abs(h) * 2.0 ** -7 + hs, 0.0)
            if odd[np.abs(h) >= np.abs(h).max() * (1 - 2.0 ** -6)].any():
                dh = np.abs(h) * 2.0 ** -6 + 2 * hs
            part = (w_down[e].astype(np.int64) @ hq[0]) * s_down[e].astype(np.float64) * hs[0]
            y[r] += w[r, j] * part
            off[r] += np.abs(w[r, j]) * (np.abs(w_down[e]).astype(np.float64) @ dh) * s_down[e]
            mag[r] += np.abs(w[r, j] * part)
    return y, off + mag * (idx.shape[1] + 6) * 2.0 ** -24, mag
