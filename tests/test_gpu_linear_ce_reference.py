"""mpt_linear_ce where the reference that a group's exponentials are taken against is at its limits: groups of classes that
are masked out altogether, and logits so large that a rounded exponent would be steps of hundreds apart."""
import numpy as np
import pytest

from gpu_util import require_gpu, torch
from test_gpu_linear_ce import H16, U, call, check, make, tc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("grads", ["none", "dW"])
@pytest.mark.parametrize("N,V", [(40, 1000), (24, 16000), (30, 40000), (300, 30000), (900, 20000)])
def test_groups_masked_by_infinite_weights(N, V, grads):
    """Classes whose first weight is -inf against a positive feature have logits of -inf and p = 0; whole groups of them must
    not take part in the row's sum even where all other logits are far below zero (here about -300).  dx is not asked for: it is
    0 * inf in that feature by its formula."""
    x, W, y = make(N, V, 64, N + V)
    x[:, 0] = 1.0 + np.arange(N) % 7
    W[:, 0] = 0.0
    x[:, 1] = 30.0
    W[:, 1] = -10.0
    masked = np.zeros(V, dtype=bool)
    masked[100:700] = True                    # four whole groups and parts of two
    masked[V - 70:] = True
    W[masked, 0] = -np.inf
    keep = np.flatnonzero(~masked)
    y = keep[np.random.default_rng(6).integers(0, len(keep), N)].astype(np.int32)
    y[3] = -1
    got = call(x, W, y, 128.0, grads)
    assert got["flag"] == 0
    if grads == "dW":
        assert not got["dW"][torch.from_numpy(masked).cuda()].any()
        got["dW"] = got["dW"][torch.from_numpy(~masked).cuda()]
    live = np.searchsorted(keep, np.where(y < 0, keep[0], y)).astype(np.int32)
    check(x, W[keep], np.where(y < 0, -1, live).astype(np.int32), 128.0, got)


@pytest.mark.parametrize("N,V", [(40, 500), (300, 20000)])
def test_rows_without_any_class_left(N, V):
    """All logits of a row -inf (or +inf, row 5): 0 / 0 (inf - inf) by the formula, so its loss is NaN."""
    x, W, y = make(N, V, 64, 7)
    x[:, 0] = 1.0
    x[5, 0] = -1.0
    W[:, 0] = -np.inf
    got = call(x, W, y, 64.0, "none")
    assert bool(got["row_loss"].isnan().all()) and np.isnan(got["loss"])


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("N,V", [(24, 700), (24, 16000), (30, 40000), (260, 20000)])
def test_logits_of_ten_billion(N, V, sign):
    """x . W = +-8 * 2^30 + 2^11 * (0..3): exact in FP32 (multiples of 2^11 below 2^34), differences of 2048 and more between
    classes, so p is 1 / (number of the row's largest logits) or 0.  d has FP16's roundings alone (normal numbers in its
    scale), losses the sum's and the logarithm's."""
    H, S = 16, 64.0
    rng = np.random.default_rng(V)
    x, W = np.zeros((N, H), dtype=np.float16), np.zeros((V, H), dtype=np.float16)
    x[:, :8], W[:, :8] = 32768.0, sign * 32768.0
    x[:, 8], W[:, 8] = 64.0, 32.0 * rng.integers(0, 3, V)
    W[rng.integers(0, V, 5), 8] = 96.0
    y = rng.integers(0, V, N).astype(np.int32)
    y[: N // 2] = rng.choice(np.flatnonzero(W[:, 8] == 96.0), N // 2)
    got = call(x, W, y, S)
    z = x.astype(np.float64) @ W.astype(np.float64).T
    m = z.max(1, keepdims=True)
    p = np.exp(z - m)
    rl = np.log(p.sum(1)) + (m[:, 0] - z[np.arange(N), y])
    p /= p.sum(1, keepdims=True)
    d = p.copy()
    d[np.arange(N), y] -= 1
    assert np.all(np.abs(got["row_loss"].cpu().numpy() - rl) <= 1e-5 + 4 * U * rl)
    e = 2 * H16 * (1 + H16) * np.abs(d) + 1e-5 * p + 2.0 ** -38
    M, X = W.astype(np.float64), x.astype(np.float64)
    c = S / N
    for name, ref, err, mag, K in (("dx", d @ M, e @ np.abs(M), np.abs(d) @ np.abs(M), V),
                                   ("dW", d.T @ X, e.T @ np.abs(X), np.abs(d).T @ np.abs(X), N)):
        g = got[name].cpu().numpy().astype(np.float64)
        t = c * (err + (tc(K) + 4 * U) * mag)
        t = t + H16 * (np.abs(c * ref) + t) + 2.0 ** -25
        fits = np.abs(c * ref) + t < 65504
        assert fits[:, 9:].all() and np.all(np.abs(g - c * ref)[fits] <= t[fits])
