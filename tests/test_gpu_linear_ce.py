"""The vocabulary head with its cross-entropy (mpt_linear_ce) against its formulas in 64 bits.

Tolerances, from the arithmetic.  u = 2^-24.  A tensor-core sum over K terms is rounded once per instruction of 16
terms and a few times inside one: (K/16 + 8) 2^-23 sum|a b| (`tc`).  A logit is off by dz = tc; a row's log-sum by at
most the largest dz of the row plus 1e-5 (sums of at most 34 terms in a chain, an exponent argument of up to 64 rounded
once, the exponential's 2 ulp: below 150 u).  p is off by p (dz_v + max dz + 1e-5) and is rounded to FP16 twice,
2^-11 of the value each time, in a scale where 2^-39 is half the smallest step; the label's p - 1 once.  The gradients' sums
take those errors times the other operand, plus their own tc, and end in one more rounding of 2^-11 (2^-25)."""
import numpy as np
import pytest

from gpu_util import require_gpu, torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
H16 = 2.0 ** -11


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def tc(K):
    return (K / 16 + 8) * 2.0 ** -23


def make(N, V, H, seed, scale=2.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((N, H)).astype(np.float16)
    W = (rng.standard_normal((V, H)) * scale / np.sqrt(H)).astype(np.float16)
    y = rng.integers(0, V, N).astype(np.int32)
    return x, W, y


def put(a, ld):
    buf = torch.full((a.shape[0], ld), float("nan"), dtype=torch.float16, device="cuda")
    buf[:, :a.shape[1]] = torch.from_numpy(a)
    return buf


def call(x, W, y, S, grads="both", row_block=0, ldx=None, ldw=None, ws=None, stream=None, out=None):
    from paper_1710_03740_b200 import binding as b
    (N, H), V = x.shape, W.shape[0]
    ldx, ldw = ldx or H, ldw or H
    xd, Wd, yd = put(x, ldx), put(W, ldw), torch.from_numpy(y).cuda()
    want_dx, want_dW = grads in ("both", "dx"), grads in ("both", "dW")
    dx = torch.full((N + 1, ldx), 7.0, dtype=torch.float16, device="cuda") if want_dx else None
    dW = torch.full((V + 1, ldw), 7.0, dtype=torch.float16, device="cuda") if want_dW else None
    rl = torch.full((N + 1,), 7.0, device="cuda")
    loss = torch.full((1,), 7.0, device="cuda")
    bad = torch.full((1,), 77, dtype=torch.int32, device="cuda")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    nbytes = b.mpt_linear_ce_workspace_bytes(N, V, H, want_dx, want_dW, row_block)
    ws = torch.full((nbytes + 256,), 0xFF, dtype=torch.uint8, device="cuda")       # every FP16 and FP32 in it a NaN
    b.mpt_linear_ce(N, V, H, xd, ldx, Wd, ldw, yd, S, rl, loss, dx, ldx, dW, ldw, ws[:nbytes], row_block, bad, flag, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert bool((ws[nbytes:] == 0xFF).all()) and float(rl[N]) == 7.0
    for g, rows in ((dx, N), (dW, V)):
        if g is not None:
            assert bool((g[rows:] == 7.0).all()) and bool((g[:, H:] == 7.0).all())     # pitch columns and the row behind
    return {"dx": None if dx is None else dx[:N, :H], "dW": None if dW is None else dW[:V, :H], "row_loss": rl[:N],
            "loss": float(loss.item()), "bad": int(bad.item()), "flag": int(flag.item())}


def check(x, W, y, S, got):
    N, H, V = x.shape[0], x.shape[1], W.shape[0]
    X, M = torch.from_numpy(x).cuda().double(), torch.from_numpy(W).cuda().double()
    yt = torch.from_numpy(y).cuda().long()
    live = (yt >= 0) & (yt < V)
    at = yt.clamp(0, V - 1)
    rows = torch.arange(N, device="cuda")
    X = torch.where(live[:, None], X, torch.zeros_like(X))          # what an ignored row holds does not count
    z = X @ M.T
    dz = (X.abs() @ M.abs().T) * tc(H)
    dzm = dz.max(1).values
    lse = torch.logsumexp(z, 1)
    rl = torch.where(live, lse - z[rows, at], torch.zeros_like(lse))
    tol = torch.where(live, dzm + dz[rows, at] + 1e-5 + 2 * U * rl.abs(), torch.zeros_like(rl))
    assert bool(((got["row_loss"].double() - rl).abs() <= tol).all())
    assert abs(got["loss"] - float(rl.mean())) <= float(tol.mean()) + 2 * U * abs(float(rl.mean())) + 1e-30
    assert got["bad"] == int((~live).sum())
    p = torch.exp(z - lse[:, None])
    pe = p * (dz + dzm[:, None] + 1e-5)
    de = pe + 2 * H16 * (1 + H16) * p + 2.0 ** -38
    d = p.clone()
    d[rows, at] -= 1.0
    de[rows, at] = (pe + H16 * d.abs())[rows, at] + 2.0 ** -38
    d = d * live[:, None]
    de = de * live[:, None]
    c = S / N
    for name, ref, err, mag, K in (("dx", d @ M, de @ M.abs(), d.abs() @ M.abs(), V), ("dW", d.T @ X, de.T @ X.abs(), d.abs().T @ X.abs(), N)):
        if got[name] is None:
            continue
        ref, t = c * ref, c * (err + (tc(K) + 4 * U) * mag)
        t = t + H16 * (ref.abs() + t) + 2.0 ** -25
        g = got[name].double()
        off = (g - ref).abs()
        assert bool((off <= t).all()), (name, float((off / t).max()), float(off.max()))


SIZES = [(1, 1, 8), (1, 2, 8), (3, 7, 16), (5, 128, 24), (64, 1000, 512), (63, 1001, 520), (128, 129, 64), (129, 257, 72),
         (300, 5003, 256), (700, 20000, 136), (257, 19001, 64), (2, 100003, 64), (130, 40000, 40), (1000, 3001, 1000),
         (300, 70001, 264), (16, 5000, 1000), (17, 129, 136), (32, 20011, 520), (33, 4099, 256), (64, 30003, 128), (65, 6001, 328),
         (128, 9001, 2048), (7, 131071, 64), (1, 40001, 4096), (1024, 200003, 1024), (2048, 70001, 2560), (2050, 33000, 1280)]


@pytest.mark.parametrize("N,V,H", SIZES)
def test_losses_and_gradients(N, V, H):
    x, W, y = make(N, V, H, N * 31 + V * 7 + H)
    S = 2.0 ** (2 + N.bit_length())
    got = call(x, W, y, S)
    check(x, W, y, S, got)
    again = call(x, W, y, S)
    assert torch.equal(got["dx"], again["dx"]) and torch.equal(got["dW"], again["dW"]) and torch.equal(got["row_loss"], again["row_loss"])


@pytest.mark.parametrize("N,V,H,row_block", [(600, 3001, 128, 256), (700, 20000, 264, 256), (513, 700, 40, 256), (1100, 260, 256, 512)])
def test_several_row_blocks(N, V, H, row_block):
    x, W, y = make(N, V, H, N + V)
    y[::9] = -1
    got = call(x, W, y, 1024.0, row_block=row_block)
    check(x, W, y, 1024.0, got)
    # one block sums the same logits, but a tile's place in the work list decides whether its k-blocks are added
    # upwards or downwards: the same bounds, not the same bits
    check(x, W, y, 1024.0, call(x, W, y, 1024.0))


@pytest.mark.parametrize("grads", ["none", "dx", "dW"])
@pytest.mark.parametrize("N,V,H", [(100, 513, 64), (400, 15000, 96), (5, 3001, 200)])
def test_parts_of_the_outputs(N, V, H, grads):
    x, W, y = make(N, V, H, 5)
    got = call(x, W, y, 512.0, grads)
    check(x, W, y, 512.0, got)


@pytest.mark.parametrize("N", [9, 200])
def test_pitched_rows(N):
    x, W, y = make(N, 777, 48, 9)
    check(x, W, y, 256.0, call(x, W, y, 256.0, ldx=64, ldw=56))


@pytest.mark.parametrize("N,V", [(50, 300), (400, 15000)])
def test_ignored_rows_may_hold_anything(N, V):
    x, W, y = make(N, V, 64, 3)
    y[[0, 7, N - 1]] = [-1, V, 2 ** 31 - 1]
    y[8] = -2 ** 31
    x[0] = np.nan
    x[7, 3] = np.inf
    x[N - 1] = 65504.0
    got = call(x, W, y, 128.0)
    check(x, W, y, 128.0, got)
    assert not got["dx"][[0, 7, 8, N - 1]].any() and got["bad"] == 4 and got["flag"] == 0


def test_all_rows_ignored():
    x, W, y = make(20, 100, 32, 3)
    y[:] = -1
    got = call(x, W, y, 128.0)
    assert got["loss"] == 0.0 and not got["dx"].any() and not got["dW"].any() and not got["row_loss"].any()


@pytest.mark.parametrize("N,V", [(40, 1000), (300, 30000)])
def test_peaked_flat_and_tiny_probabilities(N, V):
    """Rows where one class takes everything (the label's or another's), rows of equal logits, and S so small that
    p * S / N is far below what FP16 can hold: the gradients still are."""
    x, W, y = make(N, V, 64, 17)
    x[0] = 0                                                        # every p is 1 / V
    x[1] = (W[y[1]].astype(np.float32) * 40).astype(np.float16)     # the label's logit is far above the rest
    x[2] = (W[(y[2] + 1) % V].astype(np.float32) * 40).astype(np.float16)
    x[3] = -x[1]
    y[3] = y[1]
    for S in (1.0, 2.0 ** 14):
        check(x, W, y, S, call(x, W, y, S))


def test_large_logits():
    """Logits of several thousand: the exponents' reference and the sum relative to it stay apart, so p is as exact as the
    logits are.  Integer operands make every logit exact, so that the bound on d is the roundings' alone."""
    N, V, H = 24, 700, 64
    rng = np.random.default_rng(4)
    x = rng.integers(-8, 9, (N, H)).astype(np.float16) * 4
    W = rng.integers(-8, 9, (V, H)).astype(np.float16)
    x[:, :2] = 128.0
    W[:, 0] = 60.0                            # every logit is raised by 7680
    W[:, 1] = rng.integers(-3, 4, V) / 64.0
    W[:, 2:] = 0                              # what is left differs by steps of 2
    y = rng.integers(0, V, N).astype(np.int32)
    got = call(x, W, y, 64.0)
    z = x.astype(np.float64) @ W.astype(np.float64).T
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    d = p.copy()
    d[np.arange(N), y] -= 1
    # the exponents' rounding: |z log2 e| up to 2^14, rounded to 2^-10 / 2 of an exponent, but the same for one reference;
    # differences of logits are exact multiples of 2, so only the reference's own 24 bits count: (2^-10) ln 2 in the worst case
    err = np.abs(d) * 2 * H16 + p * 2.0 ** -10
    ref = (64.0 / N) * (d @ W.astype(np.float64))
    tol = (64.0 / N) * ((err + 2.0 ** -38) @ np.abs(W.astype(np.float64)) + (tc(V) + 4 * U) * (np.abs(d) @ np.abs(W.astype(np.float64))))
    assert np.all(np.abs(got["dx"].cpu().numpy() - ref) <= tol + H16 * (np.abs(ref) + tol) + 2.0 ** -25)


@pytest.mark.parametrize("N,V", [(40, 1000), (300, 30000)])
def test_classes_masked_by_their_weights(N, V):
    """Whole groups of classes whose first weight is FP16's lowest value, against a large positive feature: their logits are
    about -6e7, their p is 0, and the losses and gradients are those of the other classes alone."""
    x, W, y = make(N, V, 64, 19)
    x[:, 0] = 1000.0 + np.arange(N) / 2
    W[:, 0] = 0.0
    masked = np.zeros(V, dtype=bool)
    masked[100:700] = True
    masked[V - 70:] = True
    W[masked, 0] = -65504.0
    keep = np.flatnonzero(~masked)
    y = keep[np.random.default_rng(6).integers(0, len(keep), N)].astype(np.int32)
    got = call(x, W, y, 128.0)
    assert not got["dW"][torch.from_numpy(masked).cuda()].any() and got["flag"] == 0
    got["dW"] = got["dW"][torch.from_numpy(~masked).cuda()]
    check(x, W[keep], np.searchsorted(keep, y).astype(np.int32), 128.0, got)


@pytest.mark.parametrize("N,V", [(24, 700), (260, 20000)])
def test_logits_of_a_hundred_million(N, V):
    """x . W = 1500 * 60000 + 8 * (0..3) * 2: exact in FP32 (multiples of 8 below 2^27), differences of 16 between classes.
    FP32 spaces the exponents' reference 8 apart up there: the largest of a group is between 2^6 and 2^14, 2^-30 of it is
    kept, and differences of 16 (2^-23.08 each) are exact, so p has the roundings of FP16 (normal numbers for the largest and
    2^-24 absolute in its scale for the rest: 2^-29 of p at most)."""
    H, S = 16, 256.0
    rng = np.random.default_rng(V)
    x, W = np.zeros((N, H), dtype=np.float16), np.zeros((V, H), dtype=np.float16)
    x[:, 0], W[:, 0] = 1500.0, 60000.0
    x[:, 1], W[:, 1] = 16.0, rng.integers(0, 4, V)
    W[rng.integers(0, V, 5), 1] = 4.0
    y = rng.integers(0, V, N).astype(np.int32)
    got = call(x, W, y, S)
    z = x.astype(np.float64) @ W.astype(np.float64).T
    m = z.max(1, keepdims=True)
    p = np.exp(z - m)
    lse = m[:, 0] + np.log(p.sum(1))
    p /= p.sum(1, keepdims=True)
    d = p.copy()
    d[np.arange(N), y] -= 1
    rl = lse - z[np.arange(N), y]
    assert np.all(np.abs(got["row_loss"].cpu().numpy() - rl) <= 1e-5 + 2.0 ** -20 * rl)
    e = 2 * H16 * (1 + H16) * np.abs(d) + 1e-5 * p + 2.0 ** -28
    M, X = W.astype(np.float64), x.astype(np.float64)
    c = S / N
    for name, ref, err, mag, K in (("dx", d @ M, e @ np.abs(M), np.abs(d) @ np.abs(M), V),
                                   ("dW", d.T @ X, e.T @ np.abs(X), np.abs(d).T @ np.abs(X), N)):
        g = got[name].cpu().numpy().astype(np.float64)
        t = c * (err + (tc(K) + 4 * U) * mag)
        t = t + H16 * (np.abs(c * ref) + t) + 2.0 ** -25
        fits = np.abs(c * ref) + t < 65504
        assert fits[:, 1:].all() and np.all(np.abs(g - c * ref)[fits] <= t[fits])


def test_nonfinite_values_reach_what_they_must():
    x, W, y = make(40, 500, 64, 23)
    x[5, 1] = np.nan
    got = call(x, W, y, 64.0)
    rl = got["row_loss"].cpu().numpy()
    assert np.isnan(rl[5]) and np.isfinite(np.delete(rl, 5)).all() and np.isnan(got["loss"])
    assert bool(got["dx"][5].isnan().all()) and bool(got["dW"].isnan().all()) and got["flag"] == 1
    keep = [i for i in range(40) if i != 5]
    assert bool(got["dx"][keep].isfinite().all())


def test_overflow_of_dW_sets_the_flag():
    x, W, y = make(64, 300, 64, 29)
    got = call(x, W, y, 2.0 ** 24)
    assert got["flag"] == 1 and bool(got["dW"].isinf().any())
    assert call(x, W, y, 64.0)["flag"] == 0


def test_no_rows():
    from paper_1710_03740_b200 import binding as b
    x = torch.zeros(1, 64, dtype=torch.float16, device="cuda")
    W = torch.ones(10, 64, dtype=torch.float16, device="cuda")
    dW = torch.full((11, 64), 7.0, dtype=torch.float16, device="cuda")
    f = torch.full((1,), 7.0, device="cuda")
    loss = torch.full((1,), 7.0, device="cuda")
    y = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(b.mpt_linear_ce_workspace_bytes(0, 10, 64), dtype=torch.uint8, device="cuda")
    b.mpt_linear_ce(0, 10, 64, x, 64, W, 64, y, 1.0, f, loss, None, 64, dW, 64, ws)
    torch.cuda.synchronize()
    assert float(loss) == 0.0 and not dW[:10].any() and bool((dW[10] == 7.0).all()) and float(f) == 7.0


def test_gradients_against_differences():
    """S * d(mean loss) by central differences of the 64-bit loss: off by O(step^2) = 1e-8 and the FP16 roundings."""
    N, V, H, S, step = 4, 11, 8, 16.0, 1e-4
    x, W, y = make(N, V, H, 41)
    y[2] = -1
    got = call(x, W, y, S)
    live = (y >= 0)

    def loss(a, w):
        z = a @ w.T
        m = z.max(1, keepdims=True)
        lse = (m[:, 0] + np.log(np.exp(z - m).sum(1)))
        return S * float(((lse - z[np.arange(N), np.maximum(y, 0)]) * live).sum()) / N

    args = [x.astype(np.float64), W.astype(np.float64)]
    for k, name in enumerate(("dx", "dW")):
        num = np.zeros(args[k].shape)
        for i in np.ndindex(*num.shape):
            up, dn = [a.copy() for a in args], [a.copy() for a in args]
            up[k][i] += step
            dn[k][i] -= step
            num[i] = (loss(*up) - loss(*dn)) / (2 * step)
        g = got[name].cpu().numpy().astype(np.float64)
        # every d is within 3 * 2^-11 of its value, sums of at most 11 terms of size <= S/N * 3 each
        assert np.all(np.abs(g - num) <= 4 * H16 * (S / N) * 11 * 3)
        assert np.all(np.abs(g - num) <= 4 * H16 * np.abs(num) + 3e-2)


def test_losses_ignore_the_scale():
    x, W, y = make(70, 400, 64, 13)
    a, b = call(x, W, y, float("nan"), "none"), call(x, W, y, 1.0, "none")
    assert torch.equal(a["row_loss"], b["row_loss"]) and a["loss"] == b["loss"]


def test_captured_and_replayed():
    from paper_1710_03740_b200 import binding as b
    N, V, H, S = 300, 15000, 64, 512.0
    x, W, y = make(N, V, H, 51)
    ref = call(x, W, y, S)
    xd, Wd = torch.zeros(N, H, dtype=torch.float16, device="cuda"), torch.from_numpy(W).cuda()
    yd = torch.zeros(N, dtype=torch.int32, device="cuda")
    rl, loss = torch.empty(N, device="cuda"), torch.empty(1, device="cuda")
    dx, dW = torch.empty_like(xd), torch.empty_like(Wd)
    bad = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(b.mpt_linear_ce_workspace_bytes(N, V, H), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run = lambda: b.mpt_linear_ce(N, V, H, xd, H, Wd, H, yd, S, rl, loss, dx, H, dW, H, ws, bad_labels=bad)  # noqa: E731
        run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run()
        xd.copy_(torch.from_numpy(x))
        yd.copy_(torch.from_numpy(y))
        graph.replay()
        graph.replay()
    side.synchronize()
    assert torch.equal(dx, ref["dx"]) and torch.equal(dW, ref["dW"]) and torch.equal(rl, ref["row_loss"]) and int(bad) == 0
