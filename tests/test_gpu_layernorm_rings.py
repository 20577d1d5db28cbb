"""Layer normalisation of rows off 16-byte boundaries with many rows a warp: the buffer whose shared vector the first row
filled with ordinary stores is refilled by bulk copies several times.  Tolerances as in test_gpu_layernorm."""
import numpy as np
import pytest

from gpu_util import require_gpu
from test_gpu_layernorm import backward, forward, make, ref_backward, ref_forward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("rows,cols,ld,shift", [(40000, 131, 131, 3), (20000, 515, 515, 7), (3000, 5001, 5001, 5), (2001, 4100, 4103, 1),
                                                (30000, 100, 104, 0)])
def test_buffers_that_held_a_shared_vector(rows, cols, ld, shift):
    x, dy, gamma, beta = make(rows, cols, rows + cols)
    x[0, :8], dy[0, :8] = 30000.0, 100.0          # what a later row must not see, in the first row and behind each row's end
    x[0, -8:], dy[0, -8:] = -30000.0, -100.0
    y, mean, rstd = forward(x, gamma, beta, 1e-5, ld, shift)
    ry, _, _, tol = ref_forward(x, gamma, beta, 1e-5)
    assert np.all(np.abs(y - ry) <= tol)
    dx, dg, db, flag = backward(dy, x, gamma, mean, rstd, ld, shift)
    rdx, tdx, rdg, tdg, rdb, tdb = ref_backward(dy, x, gamma, mean, rstd)
    assert flag == 0 and np.all(np.abs(dx - rdx) <= tdx) and np.all(np.abs(dg - rdg) <= tdg) and np.all(np.abs(db - rdb) <= tdb)
