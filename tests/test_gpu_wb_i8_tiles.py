"""8-bit W_b (mla_shared_wb_i8) in each of its tiles and both output types, against 64 bits and with the device rule's own choice
asserted, so that a change of the rule cannot leave a tile without a test."""
import pytest

from test_gpu_i8 import check_wb

pytestmark = pytest.mark.gpu

# (rows, channels) of a tile and what a round of 256 of them costs
TILES = [((32 * m, 256), 6 * (m + 3), 0) for m in range(8, 1, -1)] + [((32 * m, 128), 2 * (m + 7), 0) for m in range(4, 0, -1)] + \
    [((64, 64), 10, 1), ((32, 64), 9, 1)]


def tile(n, d_out):
    if n <= 32 and -(-d_out // 16) <= 256:
        return (16 if n <= 16 else 32, 16)
    return min(TILES, key=lambda t: -(-(-(-n // t[0][0]) * -(-d_out // t[0][1])) // 256) * t[1] + t[2])[0]


# rows, channels, d_in (whole and half slices, one and many): the last rows and channels of a block ragged
CASES = {(16, 16): [(5, 203, 1088), (16, 4090, 64)], (32, 16): [(31, 2501, 192), (32, 4096, 1024)], (32, 64): [(33, 520, 704), (64, 7000, 128), (20, 6001, 64)],
         (64, 64): [(34, 12300, 192), (64, 16380, 320)], (32, 128): [(130, 6001, 448), (80, 9001, 1024)], (64, 128): [(259, 6001, 576)],
         (96, 128): [(130, 12301, 192), (192, 14000, 64)], (128, 128): [(193, 12301, 320)], (64, 256): [(259, 12300, 192), (320, 13000, 448)],
         (96, 256): [(259, 16383, 320)], (128, 256): [(385, 16380, 192)], (160, 256): [(514, 16384, 192), (2100, 4093, 576)], (192, 256): [(643, 16384, 320)],
         (224, 256): [(785, 16383, 64)], (256, 256): [(904, 16384, 192), (3709, 4090, 704)]}


def test_every_tile_has_a_case():
    assert set(CASES) == {t[0] for t in TILES} | {(16, 16), (32, 16)}


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("shape,n,d_out,d_in", [(t, *c) for t, cs in CASES.items() for c in cs])
def test_tile(shape, n, d_out, d_in, out):
    assert tile(n, d_out) == shape
    check_wb(n, d_in, d_out, out)
