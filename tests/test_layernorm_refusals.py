"""What the layer-normalisation entry points refuse, shown without a GPU: every check comes before the first CUDA call."""
import ctypes as C

import pytest

INVALID, SHAPE, WORKSPACE = -1, -2, -4
P = C.c_void_p


@pytest.fixture(scope="module")
def lib():
    from paper_1710_03740_b200 import binding, build
    build.build()
    return binding.lib()


def fwd(lib, **k):
    a = dict(rows=4, cols=64, x=P(256), ldx=64, gamma=P(512), beta=P(768), eps=1e-5, y=P(1024), ldy=64, mean=None, rstd=None, status=None, st=None)
    a.update(k)
    return lib.mpt_layernorm_forward(*a.values())


def bwd(lib, **k):
    a = dict(rows=4, cols=64, dy=P(256), lddy=64, x=P(512), ldx=64, gamma=P(768), mean=P(1024), rstd=P(1280), dx=P(1536), lddx=64,
             dgamma=P(1792), dbeta=P(2048), flag=None, status=None, ws=P(4096), nbytes=1 << 20, st=None)
    a.update(k)
    return lib.mpt_layernorm_backward(*a.values())


@pytest.mark.parametrize("change,code", [
    (dict(x=None), INVALID), (dict(gamma=None), INVALID), (dict(y=None), INVALID), (dict(y=P(256)), INVALID),
    (dict(eps=-1e-5), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(rows=-1), SHAPE), (dict(rows=(1 << 30) + 1), SHAPE), (dict(rows=2 ** 31 - 1), SHAPE), (dict(cols=0), SHAPE), (dict(ldx=63), SHAPE), (dict(ldy=63), SHAPE),
    (dict(cols=(1 << 30) + 1, ldx=(1 << 30) + 1, ldy=(1 << 30) + 1), SHAPE)])
def test_forward_refuses(lib, change, code):
    assert fwd(lib, **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(dy=None), INVALID), (dict(x=None), INVALID), (dict(gamma=None), INVALID), (dict(mean=None), INVALID),
    (dict(rstd=None), INVALID), (dict(dx=None), INVALID), (dict(dgamma=None), INVALID), (dict(ws=None), INVALID),
    (dict(dx=P(256)), INVALID), (dict(dx=P(512)), INVALID), (dict(rows=-1), SHAPE), (dict(rows=(1 << 30) + 1), SHAPE), (dict(cols=0), SHAPE), (dict(lddy=63), SHAPE),
    (dict(ldx=63), SHAPE), (dict(lddx=63), SHAPE), (dict(nbytes=4 * 64 * 8 - 1), WORKSPACE), (dict(ws=P(4100)), WORKSPACE)])
def test_backward_refuses(lib, change, code):
    assert bwd(lib, **change) == code


def test_workspace_size(lib):
    from paper_1710_03740_b200 import binding
    assert binding.mpt_layernorm_workspace_bytes(4, 64) == 4 * 64 * 8
    assert binding.mpt_layernorm_workspace_bytes(0, 1) > 0
    big = binding.mpt_layernorm_workspace_bytes(10 ** 9, 12288)
    assert big == binding.mpt_layernorm_workspace_bytes(1000, 12288) < 64 << 20          # bounded whatever the batch
    out = C.c_size_t(0)
    assert lib.mpt_layernorm_workspace_bytes(-1, 64, C.byref(out)) == SHAPE
    assert lib.mpt_layernorm_workspace_bytes((1 << 30) + 1, 64, C.byref(out)) == SHAPE
    assert lib.mpt_layernorm_workspace_bytes(4, 0, C.byref(out)) == SHAPE
    assert lib.mpt_layernorm_workspace_bytes(4, 64, None) == INVALID


def test_binding_refuses_host_tensors(lib):
    torch = pytest.importorskip("torch")
    from paper_1710_03740_b200 import binding
    t = torch.zeros(64, dtype=torch.float16)

    class FakeStream:
        device_index, cuda_stream = 0, 0

    with pytest.raises(ValueError):
        binding.mpt_layernorm_forward(1, 64, t, 64, t, None, 1e-5, t, 64, stream=FakeStream())


def test_an_empty_batch_may_come_without_addresses(lib):
    assert fwd(lib, rows=0, x=None, y=None) == 0          # nothing is launched
    assert fwd(lib, rows=0, x=None, y=None, gamma=None) == INVALID
    assert bwd(lib, rows=0, dy=None, x=None, mean=None, rstd=None, dx=None, dgamma=None) == INVALID
    assert bwd(lib, rows=0, dy=None, x=None, mean=None, rstd=None, dx=None, ws=None) == INVALID
    assert bwd(lib, rows=-1, dy=None) == INVALID and fwd(lib, rows=-1) == SHAPE
