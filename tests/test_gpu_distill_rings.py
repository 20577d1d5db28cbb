"""Distillation with many rows a CTA, where buffers whose shared vectors were mended by ordinary stores are refilled by bulk
copies again and again: the classes next to a row's ends carry its sum, so a value left over from another row would show."""
import pytest

from gpu_util import require_gpu
from test_gpu_distill import call, check, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("B,C,K,ld,shift", [(1500, 33001, 9, 33001, 3), (1200, 33001, 9, 33008, 0), (600, 70003, 5, 70003, 0), (900, 20011, 9, 20016, 0),
                                            (1500, 20001, 9, 20001, 1), (2500, 4099, 300, 4099, 5)])
def test_buffers_that_were_mended(B, C, K, ld, shift):
    z, t, idx = make(B, C, K, B + C)
    z[:, :8] += 9
    z[:, -8:] += 9
    z[::7, :8] -= 20
    z[3::7, -8:] -= 20
    S = 2.0 ** (2 + B.bit_length())
    got = call(z, t, idx, 1.0, S, ld, shift)
    check(z, t, idx, 1.0, S, got)
    check(z, t, idx, 1.0, S, call(z, t, idx, 1.0, S, ld, shift, want_dz=False))
