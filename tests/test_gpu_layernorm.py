"""Layer normalisation, forward and backward, against its formulas in 64 bits.

Tolerances.  u = 2^-24 is half a step of FP32.  A kernel's row sum passes each term through at most 64 roundings
(a thread adds at most 32 terms of its own, the rest is a tree), so it is off by at most 64 u times the sum of
absolute values; a column sum passes through at most rows / 128 + 64 of them.  Point-wise expressions add a few u of
their terms.  Rounding to FP16 adds half a step, 2^-11 of the value (2^-25 for subnormal results)."""
import numpy as np
import pytest

from gpu_util import require_gpu, torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
H16 = 2.0 ** -11
TINY = 2.0 ** -25


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def pitched(a, ld, shift=0, fill=0.0):
    """A CUDA FP16 view with row pitch ld, `shift` elements behind an aligned address, and its buffer."""
    rows, cols = a.shape
    buf = torch.full((rows * ld + shift + 8,), fill, dtype=torch.float16, device="cuda")
    view = buf[shift:shift + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(torch.from_numpy(a))
    return view, buf


def make(rows, cols, seed):
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((rows, cols)) * 1.5 + 0.3).astype(np.float16)
    dy = (rng.standard_normal((rows, cols)) * 0.25).astype(np.float16)
    gamma = (1.0 + 0.2 * rng.standard_normal(cols)).astype(np.float16)
    beta = (0.2 * rng.standard_normal(cols)).astype(np.float16)
    return x, dy, gamma, beta


def forward(x, gamma, beta, eps, ld=None, shift=0, stats=True):
    from paper_1710_03740_b200 import binding as b
    rows, cols = x.shape
    ld = cols if ld is None else ld
    xd, _ = pitched(x, ld, shift, fill=float("nan"))       # what lies between the rows must not matter
    yd, ybuf = pitched(np.zeros_like(x), ld, shift, fill=7.0)
    yd.fill_(7.0)
    gd = torch.from_numpy(gamma).cuda()
    bd = None if beta is None else torch.from_numpy(beta).cuda()
    mean = torch.full((rows,), -9.0, device="cuda") if stats else None
    rstd = torch.full((rows,), -9.0, device="cuda") if stats else None
    b.mpt_layernorm_forward(rows, cols, xd, ld, gd, bd, eps, yd, ld, mean, rstd)
    torch.cuda.synchronize()
    outside = torch.ones_like(ybuf, dtype=torch.bool)
    outside[shift:shift + rows * ld].view(rows, ld)[:, :cols] = False
    assert bool((ybuf[outside] == 7.0).all())          # between and behind the rows nothing was written
    return yd.cpu().numpy(), None if mean is None else mean.cpu().numpy(), None if rstd is None else rstd.cpu().numpy()


def backward(dy, x, gamma, mean, rstd, ld=None, shift=0, want_beta=True, ws=None):
    from paper_1710_03740_b200 import binding as b
    rows, cols = x.shape
    ld = cols if ld is None else ld
    xd, _ = pitched(x, ld, shift, fill=float("nan"))
    dyd, _ = pitched(dy, ld, shift, fill=float("nan"))
    dxd, dxbuf = pitched(np.zeros_like(x), ld, shift, fill=7.0)
    gd = torch.from_numpy(gamma).cuda()
    dg = torch.full((cols + 1,), 7.0, dtype=torch.float16, device="cuda")
    db = torch.full((cols + 1,), 7.0, dtype=torch.float16, device="cuda") if want_beta else None
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    if ws is None:
        ws = torch.full((b.mpt_layernorm_workspace_bytes(rows, cols),), 0xFF, dtype=torch.uint8, device="cuda")
    b.mpt_layernorm_backward(rows, cols, dyd, ld, xd, ld, gd, torch.from_numpy(mean).cuda(), torch.from_numpy(rstd).cuda(), dxd, ld,
                             dg, db, ws, nonfinite_flag=flag)
    torch.cuda.synchronize()
    outside = torch.ones_like(dxbuf, dtype=torch.bool)
    outside[shift:shift + rows * ld].view(rows, ld)[:, :cols] = False
    assert bool((dxbuf[outside] == 7.0).all())
    assert float(dg[cols]) == 7.0 and (db is None or float(db[cols]) == 7.0)
    return (dxd.cpu().numpy(), dg[:cols].cpu().numpy(), None if db is None else db[:cols].cpu().numpy(), int(flag.item()))


def ref_forward(x, gamma, beta, eps):
    x = x.astype(np.float64)
    mean = x.mean(1)
    var = ((x - mean[:, None]) ** 2).mean(1)
    rstd = 1.0 / np.sqrt(var + eps)
    hg = (x - mean[:, None]) * rstd[:, None] * gamma.astype(np.float64)
    bb = np.zeros(x.shape[1]) if beta is None else beta.astype(np.float64)
    tol = 64 * U * (np.abs(x).mean(1) * rstd)[:, None] * np.abs(gamma.astype(np.float64)) + 80 * U * np.abs(hg) + 4 * U * np.abs(bb)
    y = hg + bb
    return y, mean, rstd, tol + H16 * (np.abs(y) + tol) + TINY


def ref_backward(dy, x, gamma, mean, rstd):
    dy, x, gamma = dy.astype(np.float64), x.astype(np.float64), gamma.astype(np.float64)
    mean, rstd = mean.astype(np.float64)[:, None], rstd.astype(np.float64)[:, None]
    h, g = (x - mean) * rstd, dy * gamma
    c1, c2 = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
    dx = rstd * (g - c1 - h * c2)
    a1, a2 = np.abs(g).mean(1, keepdims=True), np.abs(g * h).mean(1, keepdims=True)
    tol = rstd * U * (66 * a1 + 72 * np.abs(h) * a2 + 8 * (np.abs(g) + np.abs(h * c2)))
    dx_tol = tol + H16 * (np.abs(dx) + tol) + TINY
    dg, db = (dy * h).sum(0), dy.sum(0)
    depth = x.shape[0] / 128 + 68
    gt, bt = depth * U * np.abs(dy * h).sum(0), depth * U * np.abs(dy).sum(0)
    return dx, dx_tol, dg, gt + H16 * (np.abs(dg) + gt) + TINY, db, bt + H16 * (np.abs(db) + bt) + TINY


SHAPES = [(1, 1, 1, 0), (1, 8, 8, 0), (3, 7, 7, 0), (5, 64, 64, 0), (64, 256, 256, 0), (33, 255, 256, 0), (9, 300, 301, 0),
          (150, 1000, 1000, 0), (17, 1024, 1032, 0), (1200, 1024, 1024, 0), (21, 1025, 1032, 0), (40, 2048, 2048, 0),
          (300, 4095, 4096, 0), (31, 6144, 6144, 0), (7, 6145, 6152, 0), (149, 12288, 12288, 0), (5, 12287, 12288, 0),
          (12, 1024, 1024, 3), (6, 5000, 5001, 1), (3, 12296, 12296, 0), (300, 768, 768, 0), (160, 16384, 16384, 0), (33, 15001, 15008, 0), (3, 16392, 16392, 0), (600, 8184, 8192, 0), (5, 8191, 8191, 0), (300, 2047, 2047, 0), (150, 255, 255, 1),
          (17, 12287, 12287, 5), (4, 1, 1, 3), (6, 9, 9, 1), (5, 5, 6, 7), (96, 1024, 1024, 0), (97, 1024, 1024, 0), (8, 12288, 12288, 0), (24, 4096, 4096, 0), (25, 4096, 4096, 0), (3, 9000, 9000, 0),
          (5, 6000, 6001, 1), (128, 100, 104, 0), (600, 1001, 1003, 2), (40, 16383, 16383, 0), (2, 33000, 33000, 0), (5, 40001, 40001, 1)]


@pytest.mark.parametrize("rows,cols", [(1, 3), (7, 30), (310, 1000), (9, 4099), (33, 9001)])
def test_matrices_that_lie_differently_to_16_byte_boundaries(rows, cols):
    from paper_1710_03740_b200 import binding as b
    x, dy, gamma, beta = make(rows, cols, rows + cols)
    (xd, _), (dyd, _) = pitched(x, cols + 3, 5, fill=float("nan")), pitched(dy, cols + 1, 2, fill=float("nan"))
    (yd, ybuf), (dxd, dxbuf) = pitched(np.full_like(x, 7.0), cols + 6, 1, fill=7.0), pitched(np.full_like(x, 7.0), cols + 9, 4, fill=7.0)
    gbuf = torch.zeros(cols + 3, dtype=torch.float16, device="cuda")
    gd = gbuf[3:]
    gd.copy_(torch.from_numpy(gamma))
    bd = torch.from_numpy(beta).cuda()
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dg, db = torch.empty(cols, dtype=torch.float16, device="cuda"), torch.empty(cols, dtype=torch.float16, device="cuda")
    ws = torch.empty(b.mpt_layernorm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    b.mpt_layernorm_forward(rows, cols, xd, cols + 3, gd, bd, 1e-5, yd, cols + 6, mean, rstd, status)
    b.mpt_layernorm_backward(rows, cols, dyd, cols + 1, xd, cols + 3, gd, mean, rstd, dxd, cols + 9, dg, db, ws, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    ry, _, _, tol = ref_forward(x, gamma, beta, 1e-5)
    assert np.all(np.abs(yd.cpu().numpy() - ry) <= tol)
    # the aligned call's results, to the bit: the same sums in the same order
    wy, wmean, wrstd = forward(x, gamma, beta, 1e-5, (cols + 7) // 8 * 8)
    assert np.array_equal(wy, yd.cpu().numpy()) and np.array_equal(wmean, mean.cpu().numpy()) and np.array_equal(wrstd, rstd.cpu().numpy())
    wdx, wdg, wdb, _ = backward(dy, x, gamma, wmean, wrstd, (cols + 7) // 8 * 8)
    assert np.array_equal(wdx, dxd.cpu().numpy()) and np.array_equal(wdg, dg.cpu().numpy()) and np.array_equal(wdb, db.cpu().numpy())
    for buf, ld, shift in ((ybuf, cols + 6, 1), (dxbuf, cols + 9, 4)):
        outside = torch.ones_like(buf, dtype=torch.bool)
        outside[shift:shift + rows * ld].view(rows, ld)[:, :cols] = False
        assert bool((buf[outside] == 7.0).all())


@pytest.mark.parametrize("rows,cols,ld,shift", SHAPES)
def test_forward_and_backward(rows, cols, ld, shift):
    x, dy, gamma, beta = make(rows, cols, rows * 7919 + cols)
    eps = 1e-5
    y, mean, rstd = forward(x, gamma, beta, eps, ld, shift)
    ry, rmean, rrstd, tol = ref_forward(x, gamma, beta, eps)
    assert np.all(np.abs(y - ry) <= tol)
    assert np.all(np.abs(mean - rmean) <= 66 * U * np.abs(x.astype(np.float64)).mean(1))
    # a mean that is off by d adds d^2 to the variance: far below its own rounding except where the row is constant
    dm = 66 * U * np.abs(x.astype(np.float64)).mean(1)
    assert np.all(np.abs(rstd - rrstd) <= rrstd * (40 * U + 0.5 * (dm * rrstd) ** 2))
    dx, dg, db, flag = backward(dy, x, gamma, mean, rstd, ld, shift)
    rdx, tdx, rdg, tdg, rdb, tdb = ref_backward(dy, x, gamma, mean, rstd)
    assert flag == 0
    assert np.all(np.abs(dx - rdx) <= tdx)
    assert np.all(np.abs(dg - rdg) <= tdg)
    assert np.all(np.abs(db - rdb) <= tdb)
    # again: the same bits
    dx2, dg2, db2, _ = backward(dy, x, gamma, mean, rstd, ld, shift)
    assert np.array_equal(dx, dx2) and np.array_equal(dg, dg2) and np.array_equal(db, db2)


def test_without_shift_and_without_statistics():
    x, dy, gamma, beta = make(37, 520, 5)
    y, _, _ = forward(x, gamma, None, 1e-5, stats=False)
    ry, _, _, tol = ref_forward(x, gamma, None, 1e-5)
    assert np.all(np.abs(y - ry) <= tol)
    _, mean, rstd = forward(x, gamma, None, 1e-5)
    dx, dg, db, _ = backward(dy, x, gamma, mean, rstd, want_beta=False)
    rdx, tdx, rdg, tdg, _, _ = ref_backward(dy, x, gamma, mean, rstd)
    assert db is None and np.all(np.abs(dx - rdx) <= tdx) and np.all(np.abs(dg - rdg) <= tdg)


@pytest.mark.parametrize("cols", [96, 2000])
def test_large_offset_keeps_the_variance(cols):
    """Deviations of 1 around 2000 (the spacing of FP16 there): a difference of sums of squares in FP32 would lose the
    variance of some rows altogether."""
    rng = np.random.default_rng(cols)
    x = (2000.0 + rng.integers(-2, 3, (16, cols))).astype(np.float16)
    gamma, beta = np.ones(cols, np.float16), np.zeros(cols, np.float16)
    y, mean, rstd = forward(x, gamma, beta, 0.0)
    ry, rmean, rrstd, tol = ref_forward(x, gamma, beta, 0.0)
    assert np.all(np.abs(y - ry) <= tol)
    assert np.all(np.abs(rstd / rrstd - 1.0) <= 40 * U + 0.5 * (66 * U * 2000.0 * rrstd) ** 2)


def test_special_values_stay_in_their_rows():
    x, dy, gamma, beta = make(12, 272, 11)
    x[1, 5] = np.nan
    x[2, 271] = np.inf
    x[3, :] = 4.0                 # constant: h = 0, y = beta
    x[4, :] = 65504.0
    dy[5, 3] = np.nan
    y, mean, rstd = forward(x, gamma, beta, 1e-5)
    assert np.isnan(y[1]).all() and np.isnan(y[2]).any()
    assert np.array_equal(y[3], beta) and np.array_equal(y[4], beta)
    fine = [0, 3, 4, 5, 6, 7, 8, 9, 10, 11]
    ry, _, _, tol = ref_forward(x[fine], gamma, beta, 1e-5)
    assert np.all(np.abs(y[fine] - ry) <= tol)
    dx, dg, db, flag = backward(dy, x, gamma, mean, rstd)
    assert flag == 1                                     # the NaN reaches dgamma and dbeta
    assert np.isnan(dx[1]).all() and np.isnan(dx[5]).all() and np.isnan(db[3]) and not np.isnan(db[4])
    ok = [0, 6, 7, 8, 9, 10, 11]
    rdx, tdx, *_ = ref_backward(dy[ok], x[ok], gamma, mean[ok], rstd[ok])
    assert np.all(np.abs(dx[ok] - rdx) <= tdx)


def test_overflowing_parameter_gradient_sets_the_flag():
    x, dy, gamma, _ = make(40, 64, 3)
    dy[:, 9] = 3000.0                                    # 40 * 3000 is beyond FP16
    _, mean, rstd = forward(x, gamma, None, 1e-5)
    _, _, db, flag = backward(dy, x, gamma, mean, rstd)
    assert np.isinf(db[9]) and flag == 1


def test_no_rows():
    from paper_1710_03740_b200 import binding as b
    one = torch.zeros(64, dtype=torch.float16, device="cuda")
    other = torch.zeros(64, dtype=torch.float16, device="cuda")
    f = torch.zeros(1, device="cuda")
    b.mpt_layernorm_forward(0, 64, one, 64, one, None, 1e-5, other, 64)
    dg = torch.full((64,), 7.0, dtype=torch.float16, device="cuda")
    db = torch.full((64,), 7.0, dtype=torch.float16, device="cuda")
    ws = torch.empty(b.mpt_layernorm_workspace_bytes(0, 64), dtype=torch.uint8, device="cuda")
    b.mpt_layernorm_backward(0, 64, one, 64, one, 64, one, f, f, other, 64, dg, db, ws)
    torch.cuda.synchronize()
    assert not dg.any() and not db.any()


def test_gradients_against_differences():
    """dx, dgamma and dbeta against central differences of the 64-bit forward formula."""
    rows, cols, eps = 3, 24, 1e-3
    x, dy, gamma, beta = make(rows, cols, 77)
    _, mean, rstd = forward(x, gamma, beta, eps)
    dx, dg, db, _ = backward(dy, x, gamma, mean, rstd)

    def loss(x_, g_, b_):
        m = x_.mean(1, keepdims=True)
        r = 1.0 / np.sqrt(((x_ - m) ** 2).mean(1, keepdims=True) + eps)
        return float((((x_ - m) * r * g_ + b_) * dy.astype(np.float64)).sum())

    args = [a.astype(np.float64) for a in (x, gamma, beta)]
    step = 1e-4                   # differences are off by O(step^2) = 1e-8 of third derivatives of order 1
    for k, got in enumerate((dx, dg, db)):
        num = np.zeros(args[k].shape)
        for i in np.ndindex(*args[k].shape):
            up = [a.copy() for a in args]
            dn = [a.copy() for a in args]
            up[k][i] += step
            dn[k][i] -= step
            num[i] = (loss(*up) - loss(*dn)) / (2 * step)
        assert np.all(np.abs(got - num) <= H16 * np.abs(num) + 1e-6)


def test_captured_replayed_and_on_another_stream():
    from paper_1710_03740_b200 import binding as b
    rows, cols = 500, 1536
    x, dy, gamma, beta = make(rows, cols, 21)
    y0, mean0, rstd0 = forward(x, gamma, beta, 1e-5)
    dx0, dg0, db0, _ = backward(dy, x, gamma, mean0, rstd0)
    xd, dyd = torch.zeros(rows, cols, dtype=torch.float16, device="cuda"), torch.zeros(rows, cols, dtype=torch.float16, device="cuda")
    gd, bd = torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda()
    y, dx = torch.empty_like(xd), torch.empty_like(xd)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dg, db = torch.empty_like(gd), torch.empty_like(gd)
    ws = torch.empty(b.mpt_layernorm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")

    def both(stream=None):
        b.mpt_layernorm_forward(rows, cols, xd, cols, gd, bd, 1e-5, y, cols, mean, rstd, stream=stream)
        b.mpt_layernorm_backward(rows, cols, dyd, cols, xd, cols, gd, mean, rstd, dx, cols, dg, db, ws, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            both()
        xd.copy_(torch.from_numpy(x))
        dyd.copy_(torch.from_numpy(dy))
        graph.replay()
    side.synchronize()
    assert np.array_equal(y.cpu().numpy(), y0) and np.array_equal(dx.cpu().numpy(), dx0)
    assert np.array_equal(dg.cpu().numpy(), dg0) and np.array_equal(db.cpu().numpy(), db0)
    y.zero_()
    dx.zero_()
    side.wait_stream(torch.cuda.current_stream())
    both(stream=side)             # passed in while another stream is current
    side.synchronize()
    assert np.array_equal(y.cpu().numpy(), y0) and np.array_equal(dx.cpu().numpy(), dx0)
