"""Numbers past what the kernels of the cache in 8 bits count in are refused on the host: no GPU needed."""
import pytest

import paper_2606_31315_gb300 as bp
from paper_2606_31315_gb300 import _build

P, WS, UNSUPPORTED = 0x10000, 0x20000, 2  # (addresses that nothing reads: every call here is refused)


@pytest.mark.parametrize("total", [(1 << 30) + 1, (1 << 31) - 64, (1 << 31) - 1])
@pytest.mark.parametrize("dtype", [0, 1])
def test_append_of_more_rows_than_blocks_count(total, dtype):
    """A block's first row is counted in 31 bits, up to a block past the last one."""
    _build.build()
    assert bp.load().bp_kv_append_fp8(P, P, P, P, P, 1024, P, 1024, P, P, P, 10, 64, 100, 3, total, 8, 128, dtype, WS, 256, None) == UNSUPPORTED
