"""Empty batches of the operators at the output end, as a program hands them over: tensors of no rows, whose address is null."""
import pytest

from gpu_util import require_gpu, torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def half(*shape):
    return torch.full(shape, 7.0, dtype=torch.float16, device="cuda")


def test_layer_norm():
    from paper_1710_03740_b200 import binding as b
    x, gamma, stat = half(0, 64), half(64), torch.empty(0, device="cuda")
    assert x.data_ptr() == 0
    b.mpt_layernorm_forward(0, 64, x, 64, gamma, gamma, 1e-5, half(0, 64), 64, stat, stat)
    dg, db = half(64), half(64)
    ws = torch.empty(b.mpt_layernorm_workspace_bytes(0, 64), dtype=torch.uint8, device="cuda")
    b.mpt_layernorm_backward(0, 64, x, 64, x, 64, gamma, stat, stat, half(0, 64), 64, dg, db, ws)
    torch.cuda.synchronize()
    assert not dg.any() and not db.any()


def test_head():
    from paper_1710_03740_b200 import binding as b
    x, W, dW, loss, bad = half(0, 64), half(10, 64), half(10, 64), half(1).float(), torch.ones(1, dtype=torch.int32, device="cuda")
    y, rl = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    ws = torch.empty(b.mpt_linear_ce_workspace_bytes(0, 10, 64), dtype=torch.uint8, device="cuda")
    b.mpt_linear_ce(0, 10, 64, x, 64, W, 64, y, 1.0, rl, loss, half(0, 64), 64, dW, 64, ws, bad_labels=bad)
    assert float(loss) == 0.0 and not dW.any() and int(bad) == 0


def test_distillation():
    from paper_1710_03740_b200 import binding as b
    loss = half(1).float()
    b.mpt_distill_topk(half(0, 100), 100, 0, 100, half(0, 4), torch.empty(0, 4, dtype=torch.int32, device="cuda"), 4, 4, 1.0, 1.0,
                       half(0, 100), 100, torch.empty(0, device="cuda"), loss)
    assert float(loss) == 0.0
