"""Host-side checks of the residual norms' gradient where a call has no rows (no GPU needed)."""
import os

import pytest

from test_blocks_host import NORM_GRAD, call
from test_ops_host import FAR

g = pytest.importorskip("paper_2609_29395_amd.gcpsl")

built = pytest.mark.skipif(not os.path.exists(g.LIB_PATH), reason="libgcpsl.so not built")


@built
def test_a_gradient_of_the_norm_needs_its_weights_without_rows_too():
    """The weights' gradients are written (zeros) without rows too, by a kernel that reads w_next where g_h is given."""
    for change in (dict(), dict(g_out=None), dict(r_next=None), dict(y=None, gate=None, dgate=None)):
        assert call("gcpsl_group_residual_norm_grad", NORM_GRAD, rows=0, w_next=None, dw_next=None, **change) == g.EINVAL
        assert g.lib().gcpsl_last_error()
    # nothing to write: no launch
    assert call("gcpsl_group_residual_norm_grad", NORM_GRAD, rows=0, g_h=None, dw_block=None, dw_next=None) == g.OK
    assert call("gcpsl_group_residual_norm_grad", NORM_GRAD, rows=0, g_h=FAR, dw_block=None, dw_next=None) == g.OK
