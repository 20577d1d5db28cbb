"""Layer normalisation, the vocabulary head and distillation at the ends of their documented ranges: pitches and matrices whose
offsets pass 32 bits, the longest rows and vocabularies, the largest block of rows.  Some rows of each result are held against
the formulas in 64 bits, within bounds made as in the tests of each operator."""
import pytest

from gpu_util import require_gpu, torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
H16 = 2.0 ** -11
TINY = 2.0 ** -25


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.empty_cache()


def normal(*shape, scale=1.0, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(*shape, dtype=torch.float16, device="cuda")
    for a in range(0, shape[0], max(1, (1 << 27) // max(1, out[0].numel()))):
        piece = out[a:a + max(1, (1 << 27) // max(1, out[0].numel()))]
        piece.copy_(torch.randn(piece.shape, generator=g, device="cuda") * scale)
    return out


def wide(rows, cols, pitch, fill, content=None):
    """[rows, cols] in rows `pitch` apart (the last row ends the buffer), and what must stay `fill` around them."""
    buf = torch.full(((rows - 1) * pitch + cols + 8,), fill, dtype=torch.float16, device="cuda")
    view = buf.as_strided((rows, cols), (pitch, 1))
    if content is not None:
        view.copy_(content)
    return view, buf


def untouched(buf, rows, cols, pitch, fill):
    for r in range(rows):
        gap = buf[r * pitch + cols:(r + 1) * pitch if r + 1 < rows else r * pitch + cols + 8]
        if not bool((gap[:4096] == fill).all() and (gap[-4096:] == fill).all()):
            return False
    return True


@pytest.mark.parametrize("cols,pitch", [(1000, 1 << 30), (5000, (1 << 30) + 1), (20001, (1 << 30) - 5)])
def test_layer_norm_rows_far_apart(cols, pitch):
    from paper_1710_03740_b200 import binding as b
    rows = 5
    x, _ = wide(rows, cols, pitch, float("nan"), normal(rows, cols))
    y, ybuf = wide(rows, cols, pitch, 7.0)
    gamma, beta = normal(cols, 1, seed=2)[:, 0].contiguous(), normal(cols, 1, seed=3)[:, 0].contiguous()
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    b.mpt_layernorm_forward(rows, cols, x, pitch, gamma, beta, 1e-5, y, pitch, mean, rstd)
    X, G, B = x.double(), gamma.double(), beta.double()
    m = X.mean(1, keepdim=True)
    r = ((X - m).square().mean(1, keepdim=True) + 1e-5).rsqrt()
    h = (X - m) * r
    want = h * G + B
    depth = 64 + cols / 1024          # rows of more than 12288 features: a thread adds one feature in 1024 by itself
    tol = depth * U * (X.abs().mean(1, keepdim=True) * r) * G.abs() + (depth + 16) * U * (h * G).abs() + 4 * U * B.abs()
    assert bool(((y.double() - want).abs() <= tol + H16 * (want.abs() + tol) + TINY).all()) and untouched(ybuf, rows, cols, pitch, 7.0)
    del y, ybuf
    dy, _ = wide(rows, cols, pitch, float("nan"), normal(rows, cols, seed=4))
    dx, dxbuf = wide(rows, cols, pitch, 7.0)
    dg, db = torch.empty_like(gamma), torch.empty_like(beta)
    ws = torch.empty(b.mpt_layernorm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    b.mpt_layernorm_backward(rows, cols, dy, pitch, x, pitch, gamma, mean, rstd, dx, pitch, dg, db, ws)
    D, r, h = dy.double(), rstd.double()[:, None], (X - mean.double()[:, None]) * rstd.double()[:, None]
    g = D * G
    c1, c2 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    want = r * (g - c1 - h * c2)
    tol = r * U * ((depth + 2) * g.abs().mean(1, keepdim=True) + (depth + 8) * h.abs() * (g * h).abs().mean(1, keepdim=True) + 8 * (g.abs() + (h * c2).abs()))
    assert bool(((dx.double() - want).abs() <= tol + H16 * (want.abs() + tol) + TINY).all()) and untouched(dxbuf, rows, cols, pitch, 7.0)
    for got, terms in ((dg, D * h), (db, D)):
        want, tol = terms.sum(0), 68 * U * terms.abs().sum(0)
        assert bool(((got.double() - want).abs() <= tol + H16 * (want.abs() + tol) + TINY).all())


@pytest.mark.parametrize("rows,cols", [(2, 1 << 26), (1 << 24, 3), (1 << 20, 1)])
def test_layer_norm_of_long_rows_and_of_many(rows, cols):
    from paper_1710_03740_b200 import binding as b
    x, dy = normal(rows, cols), normal(rows, cols, seed=4)
    gamma, beta = normal(cols, 1, seed=2)[:, 0].contiguous(), normal(cols, 1, seed=3)[:, 0].contiguous()
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dg, db = torch.empty_like(gamma), torch.empty_like(beta)
    ws = torch.empty(b.mpt_layernorm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    S = 1.0 / rows ** 0.5 if rows > 1000 else 1.0           # dy, so that the sums over the rows fit FP16
    dy.mul_(S)
    b.mpt_layernorm_forward(rows, cols, x, cols, gamma, beta, 1e-5, y, cols, mean, rstd)
    b.mpt_layernorm_backward(rows, cols, dy, cols, x, cols, gamma, mean, rstd, dx, cols, dg, db, ws, flag)
    X, G, B, D = x.double(), gamma.double(), beta.double(), dy.double()
    m = X.mean(1, keepdim=True)
    r = ((X - m).square().mean(1, keepdim=True) + 1e-5).rsqrt()
    depth = 64 + cols / 1024          # rows of more than 12288 features: a thread adds one feature in 1024 by itself
    h = (X - m) * r
    want = h * G + B
    # rows of few features may have next to no variance: the error of the mean, times rstd, is not small against h there
    tol = depth * U * (X.abs().mean(1, keepdim=True) * r) * (1 + h.abs()) * G.abs() + (depth + 16) * U * (h * G).abs() + 4 * U * B.abs()
    assert bool(((y.double() - want).abs() <= tol + H16 * (want.abs() + tol) + TINY).all())
    r, h = rstd.double()[:, None], (X - mean.double()[:, None]) * rstd.double()[:, None]
    g = D * G
    c1, c2 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    want = r * (g - c1 - h * c2)
    tol = r * U * ((depth + 2) * g.abs().mean(1, keepdim=True) + (depth + 8) * h.abs() * (g * h).abs().mean(1, keepdim=True) + 8 * (g.abs() + (h * c2).abs()))
    fits = want.abs() < 60000
    assert bool(((dx.double() - want).abs() <= tol + H16 * (want.abs() + tol) + TINY)[fits].all())
    down = rows / 128 + 68
    for got, terms in ((dg, D * h), (db, D)):
        want, tol = terms.sum(0), down * U * terms.abs().sum(0)
        assert bool(((got.double() - want).abs() <= tol + H16 * (want.abs() + tol) + TINY).all())
    assert int(flag) == 0


def head(N, V, H, y, x, ldx, W, ldw, dx, lddx, dW, lddw, S, row_block=0):
    from paper_1710_03740_b200 import binding as b
    rl, loss = torch.empty(N, device="cuda"), torch.empty(1, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(b.mpt_linear_ce_workspace_bytes(N, V, H, dx is not None, dW is not None, row_block), dtype=torch.uint8, device="cuda")
    b.mpt_linear_ce(N, V, H, x, ldx, W, ldw, y, S, rl, loss, dx, lddx, dW, lddw, ws, row_block, status=status)
    assert int(status) == 0
    return rl, loss


def tc(K):
    return (K / 16 + 8) * 2.0 ** -23


def head_check(N, V, H, y, x, W, dx, dW, rl, loss, S, rows, words):
    """Losses and dx of some rows (64-bit logits of those), and dW of some words (64-bit logits of all rows, in pieces).  Bounds as
    in test_gpu_linear_ce; a thread adds one group sum in 64, V / 2^13 of them, by itself."""
    pick = torch.tensor(rows, device="cuda")
    yl = y.long()

    def d_of(part):
        X = x[part].double()
        z = torch.empty(len(part), V, dtype=torch.float64, device="cuda")
        dz = torch.empty(len(part), V, dtype=torch.float64, device="cuda")
        for a in range(0, V, 1 << 20):
            M = W[a:a + (1 << 20)].double()
            z[:, a:a + (1 << 20)] = X @ M.T
            dz[:, a:a + (1 << 20)] = (X.abs() @ M.abs().T) * tc(H)
        lse = torch.logsumexp(z, 1)
        at = yl[part].clamp(0, V - 1)[:, None]
        live = ((yl[part] >= 0) & (yl[part] < V))[:, None]
        loss = (lse[:, None] - z.gather(1, at)) * live
        dzm = dz.max(1, keepdim=True).values
        off = (dzm + dz.gather(1, at) + 1e-5 + V / 2 ** 13 * U) * live + 2 * U * loss.abs()
        p = (z - lse[:, None]).exp_()
        e = p * (dz + dzm + 1e-5 + V / 2 ** 13 * U + 2 * H16 * (1 + H16)) + 2.0 ** -38
        p.scatter_add_(1, at, torch.full_like(loss, -1.0))
        e.scatter_add_(1, at, p.gather(1, at).abs() * H16)
        return p * live, e * live, loss[:, 0], off[:, 0]

    d, e, want, off = d_of(pick)
    assert bool(((rl[pick].double() - want).abs() <= off).all())
    c = S / N
    if dx is not None:
        ref, err, mag = (torch.zeros(len(rows), H, dtype=torch.float64, device="cuda") for _ in range(3))
        for a in range(0, V, 1 << 20):
            M = W[a:a + (1 << 20)].double()
            ref += d[:, a:a + (1 << 20)] @ M
            err += e[:, a:a + (1 << 20)] @ M.abs()
            mag += d[:, a:a + (1 << 20)].abs() @ M.abs()
        t = c * (err + (tc(min(V, 32768)) + (V / 32768 + 4) * U) * mag)
        assert bool(((dx[pick].double() - c * ref).abs() <= t + H16 * ((c * ref).abs() + t) + TINY).all())
    if dW is not None:
        w = torch.tensor(words, device="cuda")
        ref, err, mag = (torch.zeros(len(words), H, dtype=torch.float64, device="cuda") for _ in range(3))
        piece = max(1, (1 << 29) // V)
        for a in range(0, N, piece):
            part = torch.arange(a, min(N, a + piece), device="cuda")
            d, e, _, _ = d_of(part)
            X = x[part].double()
            ref += d[:, w].T @ X
            err += e[:, w].T @ X.abs()
            mag += d[:, w].abs().T @ X.abs()
        t = c * (err + (tc(N) + 4 * U) * mag)
        assert bool(((dW[w].double() - c * ref).abs() <= t + H16 * ((c * ref).abs() + t) + TINY).all())


@pytest.mark.parametrize("N,V,H", [(5, 70, 64), (300, 10, 264)])
def test_head_rows_far_apart(N, V, H):
    """Rows of x and dx, and of W and dW, whose offsets pass 32 bits."""
    ldx, ldw = (1 << 24, 1 << 29) if N > 100 else (1 << 30, 1 << 26)
    x, _ = wide(N, H, ldx, float("nan"), normal(N, H))
    W, _ = wide(V, H, ldw, float("nan"), normal(V, H, scale=2.0 / H ** 0.5, seed=2))
    dx, dxbuf = wide(N, H, ldx, 7.0)
    dW, dWbuf = wide(V, H, ldw, 7.0)
    y = torch.arange(N, device="cuda", dtype=torch.int32) % V
    y[1] = -1
    S = 2.0 ** (2 + N.bit_length())
    rl, loss = head(N, V, H, y, x, ldx, W, ldw, dx, ldx, dW, ldw, S)
    head_check(N, V, H, y, x, W, dx, dW, rl, loss, S, list(range(N)), list(range(V)))
    assert untouched(dxbuf, N, H, ldx, 7.0) and untouched(dWbuf, V, H, ldw, 7.0)


@pytest.mark.parametrize("N,V,H,row_block", [(3, 1 << 24, 8, 0), (260, 1 << 24, 264, 0), (3000, 793471, 64, 0), (70000, 130, 8, 65536),
                                             (70000, 1001, 72, 65536), (20000, 5003, 64, 0), (66000, 257, 16, 0)])
def test_head_of_the_largest_sizes(N, V, H, row_block):
    """The longest vocabulary, exponentials whose offsets pass 32 bits, the largest block of rows, and many default blocks."""
    x, W = normal(N, H), normal(V, H, scale=2.0 / H ** 0.5, seed=2)
    dx, dW = torch.empty_like(x), torch.empty_like(W)
    g = torch.Generator(device="cuda").manual_seed(9)
    y = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    y[N // 3] = V
    S = 2.0 ** (2 + N.bit_length())
    rl, loss = head(N, V, H, y, x, H, W, H, dx, H, dW, H, S, row_block)
    rows = sorted({0, 1, 2, N // 3, N // 2, N - 2, N - 1})
    words = sorted({0, 1, V // 2, V - 1, int(y[0]), int(y[N - 1])})
    if N * V < 1 << 33:
        head_check(N, V, H, y, x, W, dx, dW, rl, loss, S, rows, words)
    else:
        head_check(N, V, H, y, x, W, dx, None, rl, loss, S, rows, words)
    assert abs(float(loss) - float(rl.double().mean())) <= 2 * U * float(loss)


@pytest.mark.parametrize("B,C,ld,K", [(5, 700, 1 << 30, 5), (5, 20001, (1 << 30) + 3, 9), (4, 50257, (1 << 30) + 1, 9), (2, 1 << 26, 1 << 26, 20),
                                      (2, (1 << 26) - 3, (1 << 26) - 3, 1024), (5000, 500001, 500001, 4), (70000, 40000, 40000, 3), (1 << 20, 5, 5, 2)])
def test_distillation_of_the_largest_sizes(B, C, ld, K):
    from paper_1710_03740_b200 import binding as b
    far = ld > 1 << 29
    z, zbuf = wide(B, C, ld, float("nan"), normal(B, C, scale=2.0)) if far else (normal(B, C, scale=2.0), None)
    dz, buf = wide(B, C, ld, 7.0) if far else (torch.empty_like(z), None)
    t = normal(B, K, scale=2.0, seed=3)
    g = torch.Generator(device="cuda").manual_seed(5)
    idx = torch.randint(0, C, (B, K), generator=g, device="cuda", dtype=torch.int32)
    idx[0, 0] = C - 1
    rl, loss, status = torch.empty(B, device="cuda"), torch.empty(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    tau, S = 2.0, 2.0 ** (2 + B.bit_length())
    b.mpt_distill_topk(z, ld, B, C, t, idx, K, K, tau, S, dz, ld, rl, loss, status)
    assert int(status) == 0 and (buf is None or untouched(buf, B, C, ld, 7.0))
    rows = torch.tensor(sorted({0, 1, B // 3, B // 2, B - 2, B - 1} & set(range(B))), device="cuda")
    at = idx[rows].long()
    q = torch.softmax(t[rows].double() / tau, 1)
    logp = torch.log_softmax(z[rows].double() / tau, 1)
    lp = logp.gather(1, at)
    want = tau * tau * (q * (q.log() - lp)).sum(1)
    rel, relq = (C / 256 + 200) * U, (K / 32 + 200) * U
    tol = tau * tau * ((rel + relq) * 2 + (relq + 40 * U) * (q * (q.log().abs() + lp.abs())).sum(1)) + 4 * U * want.abs()
    assert bool(((rl[rows].double() - want).abs() <= tol).all())
    assert abs(float(loss) - float(rl.double().mean())) <= 2 * U * abs(float(loss))
    p = logp.exp()
    Q = torch.zeros_like(p).scatter_add_(1, at, q)
    c = tau * S / B
    e = c * ((rel + 4 * U) * p + (relq + 4 * U) * Q)
    d = c * (p - Q)
    assert bool(((dz[rows].double() - d).abs() <= e + H16 * (d.abs() + e) + TINY).all())
