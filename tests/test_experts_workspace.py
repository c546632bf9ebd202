"""The workspace of the experts (mla_moe_experts_i8_query) on the CPU: bytes that do for a number of rows do for fewer, so that a
serving loop can allocate once for its largest batch."""
import ctypes

import pytest


def _query(mla, n, d, f, e, k, dtype):
    import torch
    return mla.moe_experts_i8_query(n, d, f, e, k, torch.bfloat16 if dtype == "bf16" else torch.float32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,f,e,k", [(4096, 2048, 256, 1), (4096, 2048, 256, 8), (64, 64, 1, 1), (64, 64, 1, 16), (64, 4096, 3, 2), (4096, 64, 8, 3), (512, 1024, 32, 6),
                                     (192, 128, 1024, 16), (16384, 64, 2, 5)])
def test_never_falls_as_rows_grow(d, f, e, k, dtype):
    """Row by row across the few-pair limit of 16, around the pairs per expert where tiles get taller, around 65,536 rows, and between."""
    from paper_2609_07008_amd import mla
    near = {n + o for n in (129 * e // k, 385 * e // k, 65536, 8192 // k) for o in range(-3, 40)}
    rows = sorted({n for n in near | set(range(0, 600)) | set(range(600, 70000, 997)) if n >= 0})
    last = 0
    for n in rows:
        need = _query(mla, n, d, f, e, k, dtype)
        assert need >= last, (n, need, last)
        last = need


def test_the_call_asks_for_what_the_query_says():
    """The check of the call itself, which ends before anything is launched: a byte less than the query's is refused."""
    from paper_2609_07008_amd import mla
    for k in (1, 3, 16):
        layer = mla.MoeLayer(4096, 2048, 256, 0, k)
        a = ctypes.c_void_p(4096)
        for n in (1, 2, 5, 16, 17, 20, 300, 70000):
            own = mla.moe_experts_i8_query(n, 4096, 2048, 256, k)
            assert mla.LIB.mla_moe_experts_i8(ctypes.byref(layer), n, a, 4096, a, a, None, a, a, a, a, 0, a, a, own - 1, None) == 6   # MLA_ERR_WORKSPACE
