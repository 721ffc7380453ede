"""The largest calls of the operators on caller-owned tensors, refused on the host (no GPU needed)."""
import ctypes as C

import pytest

from test_ops_host import FAR, FORWARD, INPUT, WEIGHT, built, call, g


# The launch's threads pass 2^32, which the runtime would take modulo that: tiles of 64 x 64 by 256 threads (fp32 rows of
# few columns; few columns of a gradient), 16 x 16 (few rows of many groups), 64 x 64 by 512 (gradients), 128 x 128.
@built
@pytest.mark.parametrize("name,good,change", [
    ("gcpsl_group_forward", FORWARD, dict(rows=2 ** 30)),
    ("gcpsl_group_input_grad", INPUT, dict(rows=2 ** 30)),
    ("gcpsl_group_weight_grad", WEIGHT, dict(n=2 ** 28, k=1, lddy=2 ** 28, ldx=1, dw_gs=2 ** 28, db_gs=2 ** 28, G=4)),
    ("gcpsl_group_forward", FORWARD, dict(dtype=1, G=256, rows=256, n=2 ** 20, k=8, ldx=8, ldy=2 ** 20)),
    ("gcpsl_group_forward", FORWARD, dict(dtype=1, G=4, rows=2 ** 31 - 600, n=8, k=64, ldx=0, ldy=8)),
])
def test_launches_of_too_many_threads(name, good, change):
    assert call(name, good, **change) == g.EUNSUPPORTED


# The last rows of such tensors would pass 2^31 in a tile's or a piece's row numbers.
@built
@pytest.mark.parametrize("rows", [2 ** 31 - 1023, 2 ** 31 - 1])
@pytest.mark.parametrize("dtype", [0, 1])
def test_grouped_rows_next_to_two_to_the_31st(rows, dtype):
    size = C.c_size_t()
    assert call("gcpsl_group_forward", FORWARD, dtype=dtype, rows=rows, n=1, k=1, ldx=0, ldy=1) == g.EUNSUPPORTED
    assert call("gcpsl_group_input_grad", INPUT, dtype=dtype, rows=rows, n=1, k=1, lddy=0, lddx=1) == g.EUNSUPPORTED
    assert call("gcpsl_group_weight_grad", WEIGHT, dtype=dtype, rows=rows, n=1, k=1, lddy=0, ldx=0, workspace=FAR,
                workspace_bytes=1 << 30) == g.EUNSUPPORTED
    assert g.lib().gcpsl_group_workspace_bytes(dtype, 2, rows, 1, 1, C.byref(size)) == g.EUNSUPPORTED
    assert g.lib().gcpsl_group_workspace_bytes(dtype, 2, 2 ** 31 - 1024, 1, 1, C.byref(size)) == g.OK and size.value > 0
