"""What mpt_distill_topk refuses, shown without a GPU: every check comes before the first CUDA call."""
import ctypes as C

import pytest

INVALID, SHAPE = -1, -2
P = C.c_void_p


@pytest.fixture(scope="module")
def lib():
    from paper_1710_03740_b200 import binding, build
    build.build()
    return binding.lib()


def call(lib, **k):
    a = dict(z=P(256), ldz=64, B=4, C=64, t=P(512), idx=P(1024), ldt=8, K=8, tau=1.0, S=1.0, dz=P(2048), lddz=64, row_loss=P(4096),
             loss=P(8192), status=None, st=None)
    a.update(k)
    return lib.mpt_distill_topk(*a.values())


@pytest.mark.parametrize("change,code", [
    (dict(z=None), INVALID), (dict(t=None), INVALID), (dict(idx=None), INVALID), (dict(row_loss=None), INVALID), (dict(loss=None), INVALID),
    (dict(dz=P(256)), INVALID), (dict(tau=0.0), INVALID), (dict(tau=-1.0), INVALID), (dict(tau=float("nan")), INVALID),
    (dict(tau=float("inf")), INVALID), (dict(tau=1e-45), INVALID), (dict(tau=6e-5), INVALID), (dict(tau=16400.0), INVALID), (dict(S=float("inf")), INVALID), (dict(S=float("nan")), INVALID),
    (dict(B=-1), SHAPE), (dict(B=(1 << 30) + 1), SHAPE), (dict(B=2 ** 31 - 1), SHAPE), (dict(C=0), SHAPE), (dict(C=(1 << 26) + 1, ldz=(1 << 26) + 1, lddz=(1 << 26) + 1), SHAPE), (dict(K=0), SHAPE),
    (dict(K=1025, ldt=1025), SHAPE), (dict(ldz=63), SHAPE), (dict(lddz=63), SHAPE), (dict(ldt=7), SHAPE)])
def test_refusals(lib, change, code):
    assert call(lib, **change) == code
