"""Host-side sizes of the selective state space operators (no GPU)."""
import ctypes

import pytest

from paper_2507_04123_amd import binding as B

ROWS = sorted({*range(0, 2100, 9), *range(2100, 80000, 331), *range(80000, 900000, 7919), *(2 ** k + d for k in range(4, 31) for d in (-1, 0) if 2 ** k + d <= 2 ** 30)})


@pytest.mark.parametrize("dtype", [B.F32, B.F16, B.BF16])
@pytest.mark.parametrize("channels", [1, 3, 17, 32, 64, 90, 128, 200, 256, 520, 1024, 4097, 65536])
def test_scratch_for_more_rows_is_never_less(dtype, channels):
    """A buffer made for the largest call serves every smaller one."""
    lib = ctypes.CDLL(B.LIB_PATH)
    queries = [("emc2_causal_conv_work", (k,)) for k in (2, 4, 8)] + [("emc2_selective_scan_work", (m,)) for m in (1, 4, 16, 17, 64)]
    if channels <= 1024:
        queries.append(("emc2_gated_residual_work", ()))
    for name, more in queries:
        query = getattr(lib, name)
        query.restype, query.argtypes = ctypes.c_int64, [ctypes.c_int, ctypes.c_int64] + [ctypes.c_int32] * (1 + len(more))
        sizes = [query(dtype, n, channels, *more) for n in ROWS]
        assert min(sizes) >= 0 and sizes == sorted(sizes), (name, more)
