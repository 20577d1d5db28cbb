"""Distillation from top logits (mpt_distill_topk) against its formulas in 64 bits.

Tolerances.  u = 2^-24.  An exponential 2^x takes an argument that was rounded once (|x| u ln 2, |x| up to 64 in what
counts) and 2 ulp of its own; a row's sum adds chains of at most C / 256 + 64 terms: `rel` = (C / 256 + 200) u bounds the relative
error of the sum and of every p and q (K / 32 + 200 terms for q).  log p is off by rel + 4 u |log p|.  dz = tau S/B (p - q):
those errors of p and q, one subtraction, two multiplications, and the rounding to FP16 (2^-11 of the value, 2^-25)."""
import numpy as np
import pytest

from gpu_util import require_gpu, torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
H16 = 2.0 ** -11


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def make(B, C, K, seed):
    rng = np.random.default_rng(seed)
    z = (rng.standard_normal((B, C)) * 2).astype(np.float16)
    t = (rng.standard_normal((B, K)) * 2 + 5).astype(np.float16)
    idx = np.stack([rng.permutation(C)[:K] if K <= C else rng.integers(0, C, K) for _ in range(B)]).astype(np.int32)
    return z, t, idx


def call(z, t, idx, tau, S, ldz=None, shift=0, ldt=None, want_dz=True, stream=None):
    from paper_1710_03740_b200 import binding as b
    (B, C), K = z.shape, t.shape[1]
    ldz, ldt = ldz or C, ldt or K
    zbuf = torch.full((B * ldz + shift + 8,), float("nan"), dtype=torch.float16, device="cuda")
    zd = zbuf[shift:shift + B * ldz].view(B, ldz)
    zd[:, :C] = torch.from_numpy(z)
    td = torch.full((B, ldt), float("nan"), dtype=torch.float16, device="cuda")
    td[:, :K] = torch.from_numpy(t)
    xd = torch.zeros((B, ldt), dtype=torch.int32, device="cuda")
    xd[:, :K] = torch.from_numpy(idx)
    dzbuf = torch.full((B * ldz + shift + 8,), 7.0, dtype=torch.float16, device="cuda")
    dz = dzbuf[shift:shift + B * ldz].view(B, ldz)
    rl = torch.full((B + 1,), 7.0, device="cuda")
    loss = torch.full((1,), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    b.mpt_distill_topk(zd, ldz, B, C, td, xd, ldt, K, tau, S, dz if want_dz else None, ldz, rl, loss, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and float(rl[B]) == 7.0
    out = torch.ones_like(dzbuf, dtype=torch.bool)
    if want_dz:
        out[shift:shift + B * ldz].view(B, ldz)[:, :C] = False
    assert bool((dzbuf[out] == 7.0).all())
    return (dz[:, :C].double() if want_dz else None), rl[:B].double(), float(loss.item())


def check(z, t, idx, tau, S, got):
    dz, rl, loss = got
    B, C = z.shape
    Z = torch.from_numpy(z).cuda().double() / tau
    ix = torch.from_numpy(idx).cuda().long()
    T = torch.from_numpy(t).cuda().double() / tau
    ok = (ix >= 0) & (ix < C) & (T != -np.inf)
    live = ok.any(1)
    T = torch.where(ok, T, torch.full_like(T, -np.inf))
    q = torch.softmax(T, 1).nan_to_num(0.0)
    at = ix.clamp(0, C - 1)
    logp = torch.log_softmax(Z, 1)
    lp = logp.gather(1, at)
    terms = torch.where(q > 0, q * (torch.log(q.clamp(min=1e-300)) - lp), torch.zeros_like(q))
    ref = tau * tau * terms.sum(1)
    rel, relq = (C / 256 + 200) * U, (t.shape[1] / 32 + 200) * U
    mag = torch.where(q > 0, q * (torch.log(q.clamp(min=1e-300)).abs() + lp.abs()), torch.zeros_like(q)).sum(1)
    tol = tau * tau * ((rel + relq) * 2 + (relq + 40 * U) * mag) + 4 * U * ref.abs()
    assert bool(((rl - ref).abs() <= tol * live).all()), float(((rl - ref).abs() - tol * live).max())
    assert abs(loss - float(ref.mean())) <= float((tol * live).mean()) + 2 * U * abs(float(ref.mean()))
    if dz is None:
        return
    p = logp.exp() * live[:, None]
    Q = torch.zeros_like(p).scatter_add_(1, at, q)
    c = tau * S / B
    d = c * (p - Q)
    e = abs(c) * ((rel + 4 * U) * p + (relq + 4 * U) * Q)
    e = e + H16 * (d.abs() + e) + 2.0 ** -25
    off = (dz - d).abs()
    assert bool((off <= e).all()), float((off / e).max())


SHAPES = [  # B, C, K, pitch, shift
    (1, 1, 1, 1, 0), (2, 7, 3, 8, 0), (3, 8, 8, 8, 0), (5, 9, 2, 16, 0), (64, 1000, 8, 1000, 0), (65, 1003, 33, 1008, 0),
    (33, 1003, 5, 1003, 0), (40, 8000, 64, 8000, 3), (700, 257, 100, 264, 0), (500, 32000, 64, 32000, 0), (310, 20011, 20, 20016, 0),
    (3, 32000, 16, 32000, 0), (80, 36001, 16, 36008, 0), (160, 60000, 16, 60000, 0), (40, 100001, 1000, 100008, 0), (20, 200001, 7, 200008, 0),
    (9, 420000, 12, 420000, 0), (33, 300007, 300, 300008, 0), (20, 1000003, 50, 1000008, 0), (40, 830000, 20, 830000, 0), (40, 500009, 40, 500016, 0), (2, 793471, 128, 793472, 0), (25, 600000, 5, 600000, 1), (30, 700, 1024, 704, 0),
    (6, 400001, 1024, 400008, 0), (70, 262144, 33, 262144, 0), (3, 1, 1, 1, 5), (9, 5, 4, 5, 1), (7, 6, 3, 6, 7), (20, 13, 5, 14, 2), (300, 32001, 64, 32001, 3),
    (12, 100001, 20, 100001, 6), (5, 793471, 30, 793471, 0), (20, 50257, 9, 50259, 1), (160, 16384, 64, 16384, 0), (1000, 2048, 40, 2048, 0),
    (150, 40000, 30, 40000, 0), (151, 33001, 1024, 33001, 0), (76, 300001, 20, 300001, 0), (300, 100000, 9, 100000, 0), (3, 2050, 257, 2050, 0), (700, 64, 64, 64, 0),
    (64, 2048, 256, 2048, 0), (65, 2041, 256, 2041, 2), (40, 2047, 5, 2047, 1), (5, 16385, 300, 16385, 1)]


@pytest.mark.parametrize("B,C,K,ld,shift", SHAPES)
def test_loss_and_gradient(B, C, K, ld, shift):
    z, t, idx = make(B, C, K, B + C * 3 + K)
    tau, S = (1.0, 2.0, 4.0)[C % 3], 2.0 ** (2 + B.bit_length())
    got = call(z, t, idx, tau, S, ld, shift, K + 3)
    check(z, t, idx, tau, S, got)
    again = call(z, t, idx, tau, S, ld, shift, K + 3)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    only = call(z, t, idx, tau, S, ld, shift, K + 3, want_dz=False)
    assert torch.equal(only[1], got[1])


@pytest.mark.parametrize("C,ldz,lddz,shift", [(1003, 1008, 1003, 0), (1003, 1003, 1008, 0), (32001, 32001, 32001, 1), (5, 5, 6, 3), (800001, 800001, 800008, 0)])
def test_gradient_rows_that_lie_otherwise_than_the_logits(C, ldz, lddz, shift):
    from paper_1710_03740_b200 import binding as b
    B, K, tau, S = 9, 5, 2.0, 64.0
    z, t, idx = make(B, C, K, C + shift)
    idx[4] = -1
    ref = call(z, t, idx, tau, S)
    check(z, t, idx, tau, S, ref)
    zd = torch.full((B, ldz), float("nan"), dtype=torch.float16, device="cuda")
    zd[:, :C] = torch.from_numpy(z)
    buf = torch.full((B * lddz + shift + 8,), 7.0, dtype=torch.float16, device="cuda")
    dz = buf[shift:shift + B * lddz].view(B, lddz)
    rl, loss = torch.empty(B, device="cuda"), torch.empty(1, device="cuda")
    b.mpt_distill_topk(zd, ldz, B, C, torch.from_numpy(t).cuda(), torch.from_numpy(idx).cuda(), K, K, tau, S, dz, lddz, rl, loss)
    torch.cuda.synchronize()
    check(z, t, idx, tau, S, (dz[:, :C].double(), rl.double(), float(loss)))
    outside = torch.ones_like(buf, dtype=torch.bool)
    outside[shift:shift + B * lddz].view(B, lddz)[:, :C] = False
    assert bool((buf[outside] == 7.0).all())


@pytest.mark.parametrize("C,ld", [(50, 50), (1000, 1000), (32000, 32000), (100000, 100000), (500000, 500000)])
def test_padded_repeated_and_missing_entries(C, ld):
    B, K = 12, 40
    z, t, idx = make(B, C, K, C)
    idx[0, 5:] = -1
    idx[1, :] = -1                                   # a row without a teacher
    idx[2, ::2] = C                                  # outside on the other side
    idx[3, :] = 7                                    # one class named forty times
    idx[4, 10:20] = idx[4, 0]
    t[5, 3:] = -np.inf
    t[6, :] = -np.inf                                # entries without probability: no teacher either
    idx[7, 0], idx[7, 1] = C - 1, 0
    idx[8, 1:] = [2 ** 31 - 1, -2 ** 31] * 19 + [C]
    got = call(z, t, idx, 2.0, 64.0)
    check(z, t, idx, 2.0, 64.0, got)
    assert not got[0][1].any() and not got[0][6].any() and float(got[1][1]) == 0.0 == float(got[1][6])


@pytest.mark.parametrize("C", [300, 32000, 500000])
def test_extreme_logits(C):
    z, t, idx = make(10, C, 6, 3 + C)
    z[0, :] = 65504.0                                # equal at the type's largest value
    z[1, :] = -65504.0
    z[2, :] = -np.inf
    z[2, idx[2]] = 1.0                               # everything but the teacher's classes masked out
    z[3, :C // 2] = -np.inf
    z[3, idx[3]] = 0.5
    z[4, 17] = 60000.0                               # one class takes everything
    z[5, :] = -65504.0
    z[5, idx[5, 0]] = 0.0
    t[6, :] = [65504.0, -65504.0, 0, 0, 0, 0]
    check(z, t, idx, 1.0, 64.0, call(z, t, idx, 1.0, 64.0))


@pytest.mark.parametrize("C", [300, 32000, 500000])
def test_smallest_temperature(C):
    """tau = 2^-14: exponents of up to 1.5e9, which FP32 spaces 128 apart.  Logits that differ do so by at least 2^-9 / tau = 32,
    so every p is 1 / (number of the row's largest logits) or below e^-32, and so is q."""
    B, K, tau, S = 6, 5, 2.0 ** -14, 2.0 ** 20
    rng = np.random.default_rng(C)
    z, t, idx = make(B, C, K, 77 + C)
    z = (rng.integers(-65504 // 32, 65504 // 32 + 1, (B, C)) * 32.0).astype(np.float16)
    t = rng.integers(-8, 9, (B, K)).astype(np.float16)
    z[1] = -65504.0
    z[2, 5] = 65504.0
    z[3] = np.where(np.arange(C) % 3 == 0, 65472.0, -65504.0)
    z[4] = 1.5 - rng.integers(0, 2, C) / 512.0
    dz, rl, loss = call(z, t, idx, tau, S)
    top = z == z.max(1, keepdims=True)
    p = top / top.sum(1, keepdims=True)
    tt = t == t.max(1, keepdims=True)
    q = tt / tt.sum(1, keepdims=True)
    d = p.copy()
    for r in range(B):
        np.add.at(d[r], idx[r], -q[r])
    c = tau * S / B
    rel = (C / 256 + 200 + K) * U
    e = c * ((rel + 2.0 ** -46) * (np.abs(d) + 2 * p) + 2.0 ** -46)
    e = e + H16 * (np.abs(c * d) + e) + 2.0 ** -25
    assert np.all(np.abs(dz.cpu().numpy() - c * d) <= e)
    assert np.isfinite(loss) and bool(rl.isfinite().all())


@pytest.mark.parametrize("C", [300, 32000, 500000])
def test_nonfinite_values_stay_in_their_rows(C):
    z, t, idx = make(8, C, 6, 5 + C)
    z[1, 3] = np.nan
    z[2, C - 1] = np.inf
    z[3, :] = -np.inf
    t[4, 2] = np.nan
    z[5, :] = np.nan
    z[6, idx[6, 1]] = -np.inf                        # a class the teacher wants and the student excludes: infinite loss
    dz, rl, loss = call(z, t, idx, 1.0, 64.0)
    rl = rl.cpu().numpy()
    assert np.isnan(rl[[1, 2, 3, 4, 5]]).all() and np.isposinf(rl[6]) and np.isfinite(rl[[0, 7]]).all() and not np.isfinite(loss)
    assert bool(dz[[1, 2, 3, 5]].isnan().all()) and bool(dz[4][idx[4].tolist()].isnan().all())
    assert bool(dz[[0, 6, 7]].isfinite().all())
    keep = [0, 7]
    check(z[keep], t[keep], idx[keep], 1.0, 16.0, (dz[keep], torch.from_numpy(rl[keep]).cuda(), float(rl[keep].mean())))   # 64 / 8 = 16 / 2


def test_no_rows():
    from paper_1710_03740_b200 import binding as b
    z = torch.zeros(8, dtype=torch.float16, device="cuda")
    dz = torch.full((8,), 7.0, dtype=torch.float16, device="cuda")
    i = torch.zeros(8, dtype=torch.int32, device="cuda")
    rl, loss = torch.full((1,), 7.0, device="cuda"), torch.full((1,), 7.0, device="cuda")
    b.mpt_distill_topk(z, 8, 0, 8, z, i, 4, 4, 1.0, 1.0, dz, 8, rl, loss)
    torch.cuda.synchronize()
    assert float(loss) == 0.0 and float(rl) == 7.0 and bool((dz == 7.0).all())


def test_gradient_against_differences():
    """S * d(mean loss)/dz by central differences of the 64-bit loss (off by O(step^2) = 1e-8) and the FP16 rounding."""
    B, C, K, tau, S, step = 3, 13, 4, 2.0, 8.0, 1e-4
    z, t, idx = make(B, C, K, 99)
    idx[1, 2] = -1
    idx[2, 1] = idx[2, 0]
    dz, _, _ = call(z, t, idx, tau, S)
    ok = idx >= 0
    T = np.where(ok, t.astype(np.float64) / tau, -np.inf)
    q = np.exp(T - T.max(1, keepdims=True))
    q /= q.sum(1, keepdims=True)

    def loss(zz):
        zz = zz / tau
        lp = zz - np.log(np.exp(zz).sum(1, keepdims=True))
        l = np.where(ok, q * (np.log(np.where(ok, q, 1.0)) - np.take_along_axis(lp, np.maximum(idx, 0), 1)), 0.0)
        return S * tau * tau * l.sum() / B

    z64 = z.astype(np.float64)
    num = np.zeros_like(z64)
    for i in np.ndindex(*z64.shape):
        up, dn = z64.copy(), z64.copy()
        up[i] += step
        dn[i] -= step
        num[i] = (loss(up) - loss(dn)) / (2 * step)
    assert np.all(np.abs(dz.cpu().numpy() - num) <= 2 * H16 * np.abs(num) + 1e-5)


def test_captured_and_replayed():
    from paper_1710_03740_b200 import binding as b
    B, C, K, tau, S = 200, 32000, 16, 2.0, 512.0
    z, t, idx = make(B, C, K, 8)
    ref = call(z, t, idx, tau, S)
    zd = torch.zeros(B, C, dtype=torch.float16, device="cuda")
    td, xd = torch.from_numpy(t).cuda(), torch.from_numpy(idx).cuda()
    dz, rl, loss = torch.empty_like(zd), torch.empty(B, device="cuda"), torch.empty(1, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run = lambda: b.mpt_distill_topk(zd, C, B, C, td, xd, K, K, tau, S, dz, C, rl, loss)  # noqa: E731
        run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run()
        zd.copy_(torch.from_numpy(z))
        graph.replay()
        graph.replay()
    side.synchronize()
    assert torch.equal(dz.double(), ref[0]) and torch.equal(rl.double(), ref[1])
