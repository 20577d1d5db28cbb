"""mpt_linear_ce over long contractions and many rows: how far dx's sums may drift, and several blocks of rows whose dx is cut
into parts or launches.  (Tolerances of the second as in test_gpu_linear_ce.)"""
import math

import pytest

from gpu_util import require_gpu, torch
from test_gpu_linear_ce import H16, U, call, check, make, tc

pytestmark = pytest.mark.gpu

PART = 32768          # terms that one accumulator of dx takes at most


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("N,V,H", [(1024, 1 << 19, 1024), (300, 1 << 19, 264), (128, 1 << 19, 1024), (2048, 1 << 19, 2560), (200, 1 << 18, 18944)])
def test_no_accumulator_of_dx_drifts(N, V, H):
    """x = 0, so every p is 1 / V, exactly (V a power of two), and with W positive, and zero for the label's class, dx is the mean
    of a column of W times S / N: terms of one sign, whose sum in one accumulator loses part of a step towards zero at each of its
    K / 16 additions.  One accumulator takes at most PART terms (relative error tc(PART)), adding the parts one rounding each.  The mean
    over the columns, which lie anywhere in a factor of two, takes the rounding to FP16 out but for 6 standard deviations of
    2^-11 / sqrt(3 H).  One accumulator over all V terms would lose some 2^-25 * V / 16, 5e-4 to 1e-3."""
    from paper_1710_03740_b200 import binding as b
    g = torch.Generator(device="cuda").manual_seed(H + N)
    scale = 2.0 ** torch.rand(H, generator=g, device="cuda")
    W = torch.empty(V, H, dtype=torch.float16, device="cuda")
    for a in range(0, V, 1 << 16):
        W[a:a + (1 << 16)] = ((0.5 + 0.5 * torch.rand(1 << 16, H, generator=g, device="cuda")) * scale).half()
    W[0] = 0
    x, y = torch.zeros(N, H, dtype=torch.float16, device="cuda"), torch.zeros(N, dtype=torch.int32, device="cuda")
    rl, loss, dx = torch.empty(N, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(x)
    ws = torch.empty(b.mpt_linear_ce_workspace_bytes(N, V, H, True, False), dtype=torch.uint8, device="cuda")
    b.mpt_linear_ce(N, V, H, x, H, W, H, y, 4.0 * N, rl, loss, dx, H, None, H, ws)
    total = torch.zeros(H, dtype=torch.float64, device="cuda")
    for a in range(0, V, 1 << 16):
        total += W[a:a + (1 << 16)].double().sum(0)
    off = dx.double() / (4.0 * total / V) - 1.0
    assert bool(((rl.double() - math.log(V)).abs() <= 1e-5).all())
    drift = tc(PART) + V / PART * U
    assert bool((off.abs() <= drift + H16 * (1 + drift)).all())
    assert float(off.mean(1).abs().max()) <= drift + 6 * H16 / math.sqrt(3 * H), float(off.mean())


@pytest.mark.parametrize("N,V,H,row_block", [(1100, 40000, 264, 512), (2304, 70001, 2560, 2048), (600, 33001, 520, 256), (4500, 9001, 136, 0),
                                             (4097, 40000, 72, 0)])
def test_row_blocks_with_long_contractions(N, V, H, row_block):
    x, W, y = make(N, V, H, N + V)
    y[::9] = -1
    S = 2.0 ** (2 + N.bit_length())
    check(x, W, y, S, call(x, W, y, S, row_block=row_block))


@pytest.mark.parametrize("N,V,H", [(64, 1000, 512), (200, 3001, 264), (300, 33001, 264), (512, 70000, 64)])
def test_a_factor_of_one(N, V, H):
    """S / N * 2^-14 = 1: the products then take the kernels of ordinary calls where nothing else is asked of them.  A gradient may
    be beyond FP16 here (16384 |x| for a label's word, |x| > 4): infinite then, with its sign."""
    x, W, y = make(N, V, H, N + V, scale=0.5)
    got = call(x, W, y, 16384.0 * N)
    X, M, at = torch.from_numpy(x).cuda().double(), torch.from_numpy(W).cuda().double(), torch.from_numpy(y).cuda().long()
    d = torch.softmax(X @ M.T, 1)
    d[torch.arange(N, device="cuda"), at] -= 1.0
    for name, ref in (("dx", 16384.0 * (d @ M)), ("dW", 16384.0 * (d.T @ X))):
        over = got[name].isinf()
        assert bool((ref[over].abs() >= 65504.0 * (1 - 4 * H16)).all()) and bool((ref[over].sign() == got[name][over].sign()).all())
        got[name] = torch.where(over, ref, got[name].double())
    check(x, W, y, 16384.0 * N, got)
