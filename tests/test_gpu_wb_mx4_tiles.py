"""4-bit W_b (mla_shared_wb_mx4) in each of its tiles and both output types, against 64 bits and
with the device rule's own choice asserted, so that a change of the rule cannot leave a tile
without a test."""
import numpy as np
import pytest

import mx4_reference as R
from test_gpu_mx4 import _bf16_dev, _host, _wb, _weight

pytestmark = pytest.mark.gpu

TILES = [(16, 16), (32, 16), (16, 32), (32, 32), (16, 64), (32, 64), (64, 64), (64, 128)]


def tile(n, d_out):
    """(rows, channels) of the tile that the library takes: rounds over the 256 units, each by what it costs."""
    def cost(t):
        blocks = -(-n // t[0]) * -(-d_out // t[1])
        return -(-blocks // 256) * (5 * min(n, t[0]) + 8 * t[1] + 80)
    return min((t for t in TILES if t[0] == 16 or t[0] // 2 < n), key=cost)


# rows, channels, d_in: the last rows and channels of a block ragged, one row block and several
CASES = {(16, 16): [(5, 203, 1088), (33, 77, 448)], (32, 16): [(31, 2501, 192), (32, 4096, 576), (17, 2101, 64)],
         (16, 32): [(9, 6151, 320)], (32, 32): [(30, 6153, 192)], (16, 64): [(9, 12301, 448)], (32, 64): [(30, 12302, 320)],
         (64, 64): [(190, 12301, 192), (40, 12300, 576)], (64, 128): [(150, 6151, 320)]}


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("shape,n,d_out,d_in", [(t, *c) for t, cs in CASES.items() for c in cs])
def test_tile(shape, n, d_out, d_in, out):
    import torch
    assert tile(n, d_out) == shape
    rng = np.random.default_rng(n + d_in + d_out)
    z = _bf16_dev(rng.standard_normal((n, d_in)))
    c, s = _weight(d_out, d_in, d_in + d_out)
    y = _wb(z, c, s, out)
    w, zz = R.values(c, s), _host(z)
    want = zz @ w.T
    # at most d_in half steps 2^-24 of the sum of magnitudes; half a step of a bf16 output
    bound = d_in * 2.0 ** -24 * (np.abs(zz) @ np.abs(w).T) + 1e-30
    if out == "bf16":
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    assert (np.abs(_host(y) - want) <= bound).all()
    bits = torch.int16 if out == "bf16" else torch.int32
    for row in (0, n - 1):
        assert torch.equal(_wb(z[row:row + 1].contiguous(), c, s, out).view(bits), y[row:row + 1].view(bits))
