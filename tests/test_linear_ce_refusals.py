"""What mpt_linear_ce refuses, shown without a GPU: every check comes before the first CUDA call."""
import ctypes as C

import pytest

INVALID, SHAPE, WORKSPACE = -1, -2, -4
P = C.c_void_p


@pytest.fixture(scope="module")
def lib():
    from paper_1710_03740_b200 import binding, build
    build.build()
    return binding.lib()


def call(lib, **k):
    a = dict(N=4, V=10, H=64, x=P(256), ldx=64, W=P(512), ldw=64, labels=P(1024), S=1.0, row_block=0, dx=P(2048), lddx=64, dW=P(4096),
             lddw=64, row_loss=P(8192), loss=P(12288), bad=None, flag=None, status=None, ws=P(1 << 16), nbytes=1 << 30, st=None)
    a.update(k)
    return lib.mpt_linear_ce(*a.values())


@pytest.mark.parametrize("change,code", [
    (dict(x=None), INVALID), (dict(W=None), INVALID), (dict(labels=None), INVALID), (dict(row_loss=None), INVALID),
    (dict(loss=None), INVALID), (dict(ws=None), INVALID), (dict(S=float("nan")), INVALID), (dict(S=float("inf")), INVALID),
    (dict(dx=P(256)), INVALID), (dict(dW=P(512)), INVALID),
    (dict(N=-1), SHAPE), (dict(N=(1 << 30) + 1), SHAPE), (dict(N=2 ** 31 - 1), SHAPE), (dict(H=(1 << 30) + 8, ldx=(1 << 30) + 8, ldw=(1 << 30) + 8), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 24) + 1), SHAPE), (dict(H=0), SHAPE), (dict(H=60), SHAPE), (dict(row_block=-256), SHAPE),
    (dict(row_block=100), SHAPE), (dict(row_block=65536 + 256), SHAPE), (dict(ldx=56), SHAPE), (dict(ldw=56), SHAPE), (dict(lddx=56), SHAPE), (dict(lddw=56), SHAPE),
    (dict(ldx=68), SHAPE), (dict(ldw=68), SHAPE), (dict(lddx=68), SHAPE), (dict(lddw=68), SHAPE), (dict(x=P(264)), SHAPE),
    (dict(W=P(520)), SHAPE), (dict(dx=P(2056)), SHAPE), (dict(dW=P(4104)), SHAPE),
    (dict(nbytes=100), WORKSPACE), (dict(ws=P((1 << 16) + 16)), WORKSPACE)])
def test_refusals(lib, change, code):
    assert call(lib, **change) == code


def test_workspace_size(lib):
    from paper_1710_03740_b200 import binding as b
    full = b.mpt_linear_ce_workspace_bytes(4096, 32000, 1024)
    assert full >= 4096 * 32000 * 2
    # losses alone need no exponentials; row blocks bound the rest whatever N is
    assert b.mpt_linear_ce_workspace_bytes(4096, 32000, 1024, False, False) < full / 8
    assert b.mpt_linear_ce_workspace_bytes(10 ** 6, 32000, 1024, True, False, 512) < full / 4
    blocks = b.mpt_linear_ce_workspace_bytes(10 ** 6, 32000, 1024, True, True, 512)
    assert 32000 * 1024 * 4 < blocks < 32000 * 1024 * 4 + full / 4
    with pytest.raises(b.MptError):
        b.mpt_linear_ce_workspace_bytes(16, 32000, 1020)
    out = C.c_size_t(0)
    assert lib.mpt_linear_ce_workspace_bytes(4, 10, 64, 1, 1, 0, None) == INVALID
    assert lib.mpt_linear_ce_workspace_bytes(2 ** 31 - 1, 10, 64, 1, 1, 0, C.byref(out)) == SHAPE
    assert b.mpt_linear_ce_workspace_bytes(1 << 30, 10, 64) == b.mpt_linear_ce_workspace_bytes(8192, 10, 64)
    assert lib.mpt_linear_ce_workspace_bytes(4, 10, 64, 1, 1, 255, C.byref(out)) == SHAPE
