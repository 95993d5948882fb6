"""Host-side sizes of the sequence operators (no GPU)."""
import ctypes

import pytest

from paper_2507_04123_amd import binding as B

ROWS = sorted({*range(0, 2100, 9), *range(2100, 80000, 331), *range(80000, 900000, 7919), *(2 ** k + d for k in range(4, 31) for d in (-1, 0) if 2 ** k + d <= 2 ** 30)})


@pytest.mark.parametrize("dtype", [B.F32, B.F16, B.BF16])
@pytest.mark.parametrize("channels", [1, 3, 17, 32, 64, 90, 128, 200, 256])
def test_scratch_for_more_rows_is_never_less(dtype, channels):
    """A buffer made for the largest call serves every smaller one."""
    lib = ctypes.CDLL(B.LIB_PATH)
    for name, hidden in (("emc2_layernorm_work", ()), ("emc2_recurrence_work", ()), *(("emc2_ffn_work", (h,)) for h in (8, 40, 200, 256, 384, 1024, 9000, 65536))):
        query = getattr(lib, name)
        query.restype, query.argtypes = ctypes.c_int64, [ctypes.c_int, ctypes.c_int64] + [ctypes.c_int32] * (1 + len(hidden))
        sizes = [query(dtype, n, channels, *hidden) for n in ROWS]
        assert min(sizes) >= 0 and sizes == sorted(sizes), (name, hidden)
