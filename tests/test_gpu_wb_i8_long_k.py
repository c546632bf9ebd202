"""8-bit W_b (mla_shared_wb_i8) in each of its tiles with K of more than twice the slices that the tile keeps in LDS, so that its
loop refills every one of them and wraps around: a whole last slice and a half one, both output types, against 64 bits.  That
the sizes do so is asserted on the CPU, of the library's own rule (test_i8_rules.py)."""
import pytest

from test_gpu_i8 import check_wb

pytestmark = pytest.mark.gpu

# tile: rows and channels that get it, and d_in
CASES = {(16, 16): (7, 203, (9216, 9280)), (32, 16): (31, 330, (7168, 7232)), (32, 64): (33, 520, (1664, 1728)), (64, 64): (34, 12300, (1408, 1472)),
         (32, 128): (130, 6001, (1920, 1984)), (64, 128): (259, 6001, (1664, 1728)), (96, 128): (130, 12301, (1408, 1472)), (128, 128): (193, 12301, (1152, 1216)),
         (64, 256): (259, 12300, (896, 960)), (96, 256): (259, 16383, (896, 960)), (128, 256): (385, 16380, (896, 960)), (160, 256): (514, 16384, (896, 960)),
         (192, 256): (643, 16384, (640, 704)), (224, 256): (785, 16383, (640, 704)), (256, 256): (904, 16384, (640, 704))}


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("n,d_out,d_in", [(n, d_out, d_in) for n, d_out, ds in CASES.values() for d_in in ds])
def test_tile(n, d_out, d_in, out):
    check_wb(n, d_in, d_out, out)


def test_listed_depths():
    """K of 4096 and 7168 in tiles of each height of 128 and 256 channels, as layers have them."""
    for n, d_in, d_out in ((200, 4096, 7168), (300, 7168, 4096), (1000, 4096, 4096), (2100, 7168, 4096), (4096, 4096, 4000)):
        check_wb(n, d_in, d_out, "bf16")
