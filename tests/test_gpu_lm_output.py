"""The output end of a language model as a program runs it: final normalisation, vocabulary head with its loss (or logits
and distillation), back through the normalisation, and the master pass on the gradients.  Every stage is held to its
formula in 64 bits on the inputs it was really given, with the tolerances of the operators' own tests; the chain's end
is also compared with 64-bit autograd through the whole of it."""
import numpy as np
import pytest

from gpu_util import require_gpu, torch
import test_gpu_distill
import test_gpu_layernorm
import test_gpu_linear_ce

pytestmark = pytest.mark.gpu

EPS = 1e-5
H16 = 2.0 ** -11


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


class Chain:
    """Buffers and calls of norm -> head + loss -> norm backward, N rows of H features, V words."""

    def __init__(self, N, H, V, seed, S):
        from paper_1710_03740_b200 import binding as b
        self.b, self.N, self.H, self.V, self.S = b, N, H, V, S
        rng = np.random.default_rng(seed)
        self.h = (rng.standard_normal((N, H)) * 1.5 + 0.2).astype(np.float16)
        self.gamma = (1 + 0.1 * rng.standard_normal(H)).astype(np.float16)
        self.beta = (0.1 * rng.standard_normal(H)).astype(np.float16)
        self.W = (rng.standard_normal((V, H)) * 2 / np.sqrt(H)).astype(np.float16)
        self.y = rng.integers(0, V, N).astype(np.int32)
        self.y[::7] = -1
        c = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
        e = lambda *s, t=torch.float16: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
        f = torch.float32
        self.hd, self.gd, self.bd, self.Wd, self.yd = c(self.h), c(self.gamma), c(self.beta), c(self.W), c(self.y)
        self.x, self.mean, self.rstd = e(N, H), e(N, t=f), e(N, t=f)
        self.row_loss, self.loss = e(N, t=f), e(1, t=f)
        self.dx, self.dW, self.dh, self.dg, self.db = e(N, H), e(V, H), e(N, H), e(H), e(H)
        self.flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws_ce = e(b.mpt_linear_ce_workspace_bytes(N, V, H), t=torch.uint8)
        self.ws_ln = e(b.mpt_layernorm_workspace_bytes(N, H), t=torch.uint8)

    def run(self):
        b, N, H, V = self.b, self.N, self.H, self.V
        b.mpt_layernorm_forward(N, H, self.hd, H, self.gd, self.bd, EPS, self.x, H, self.mean, self.rstd, status=self.status)
        b.mpt_linear_ce(N, V, H, self.x, H, self.Wd, H, self.yd, self.S, self.row_loss, self.loss, self.dx, H, self.dW, H, self.ws_ce,
                        nonfinite_flag=self.flag, status=self.status)
        b.mpt_layernorm_backward(N, H, self.dx, H, self.hd, H, self.gd, self.mean, self.rstd, self.dh, H, self.dg, self.db, self.ws_ln,
                                 nonfinite_flag=self.flag, status=self.status)

    def outputs(self):
        return [t.clone() for t in (self.x, self.mean, self.rstd, self.row_loss, self.loss, self.dx, self.dW, self.dh, self.dg, self.db)]


@pytest.mark.parametrize("N,H,V", [(1, 64, 50), (96, 256, 1003), (300, 520, 9000), (640, 1024, 32000)])
def test_norm_head_loss_and_back(N, H, V):
    S = 2.0 ** (2 + N.bit_length())
    c = Chain(N, H, V, N + V, S)
    if N == 1:
        c.yd.fill_(3)
        c.y[:] = 3
    c.run()
    torch.cuda.synchronize()
    assert int(c.flag) == 0 and int(c.status) == 0
    x = c.x.cpu().numpy()
    ry, _, _, tol = test_gpu_layernorm.ref_forward(c.h, c.gamma, c.beta, EPS)
    assert np.all(np.abs(x - ry) <= tol)
    test_gpu_linear_ce.check(x, c.W, c.y, S, {"row_loss": c.row_loss, "loss": float(c.loss), "bad": int((c.y < 0).sum()), "dx": c.dx, "dW": c.dW})
    rdx, tdx, rdg, tdg, rdb, tdb = test_gpu_layernorm.ref_backward(c.dx.cpu().numpy(), c.h, c.gamma, c.mean.cpu().numpy(), c.rstd.cpu().numpy())
    assert np.all(np.abs(c.dh.cpu().numpy() - rdx) <= tdx)
    assert np.all(np.abs(c.dg.cpu().numpy() - rdg) <= tdg) and np.all(np.abs(c.db.cpu().numpy() - rdb) <= tdb)
    # end to end, 64-bit autograd.  Roundings on the way to any gradient: x (2^-11 of each element, which moves p by that of a
    # logit), d twice, dx once, the result once; the normalisation's backward pass adds no more than twice what comes in.
    # 16 half steps bound their sum in norm.
    h = torch.from_numpy(c.h).cuda().double().requires_grad_()
    g = torch.from_numpy(c.gamma).cuda().double().requires_grad_()
    bt = torch.from_numpy(c.beta).cuda().double().requires_grad_()
    W = torch.from_numpy(c.W).cuda().double().requires_grad_()
    xx = torch.nn.functional.layer_norm(h, (H,), g, bt, EPS)
    loss = torch.nn.functional.cross_entropy(xx @ W.T, c.yd.long(), ignore_index=-1, reduction="sum") / N
    (loss * S).backward()
    total = float(loss.detach())
    assert abs(float(c.loss) - total) <= 4 * H16 * total
    for got, ref in ((c.dh, h.grad), (c.dW, W.grad), (c.dg, g.grad), (c.db, bt.grad)):
        assert float((got.double() - ref).norm()) <= 16 * H16 * float(ref.norm())


def test_norm_logits_distillation_and_back():
    """The same with logits from the framework's own product and a teacher instead of labels."""
    from paper_1710_03740_b200 import binding as b
    N, H, V, K, tau = 200, 256, 5000, 24, 2.0
    S = 1024.0
    c = Chain(N, H, V, 5, S)
    rng = np.random.default_rng(6)
    t = (rng.standard_normal((N, K)) * 2 + 4).astype(np.float16)
    idx = np.stack([rng.permutation(V)[:K] for _ in range(N)]).astype(np.int32)
    idx[::11] = -1
    z = torch.empty(N, V, dtype=torch.float16, device="cuda")
    dz = torch.empty_like(z)
    b.mpt_layernorm_forward(N, H, c.hd, H, c.gd, c.bd, EPS, c.x, H, c.mean, c.rstd)
    b.mpt_gemm_f16(b.OP_FWD, N, V, H, c.x, H, c.Wd, H, z, V)
    b.mpt_distill_topk(z, V, N, V, torch.from_numpy(t).cuda(), torch.from_numpy(idx).cuda(), K, K, tau, S, dz, V, c.row_loss, c.loss, c.status)
    b.mpt_gemm_f16(b.OP_DGRAD, N, H, V, dz, V, c.Wd, H, c.dx, H)
    b.mpt_gemm_f16(b.OP_WGRAD, V, H, N, dz, V, c.x, H, c.dW, H, nonfinite_flag=c.flag)
    b.mpt_layernorm_backward(N, H, c.dx, H, c.hd, H, c.gd, c.mean, c.rstd, c.dh, H, c.dg, c.db, c.ws_ln, nonfinite_flag=c.flag)
    torch.cuda.synchronize()
    assert int(c.flag) == 0 and int(c.status) == 0
    test_gpu_distill.check(z.cpu().numpy(), t, idx, tau, S, (dz.double(), c.row_loss.double(), float(c.loss)))
    rdx, tdx, rdg, tdg, rdb, tdb = test_gpu_layernorm.ref_backward(c.dx.cpu().numpy(), c.h, c.gamma, c.mean.cpu().numpy(), c.rstd.cpu().numpy())
    assert np.all(np.abs(c.dh.cpu().numpy() - rdx) <= tdx)
    # without a teacher a row gives no gradient at all
    assert not c.dh[::11].any()


def test_training_lowers_nothing_but_runs_and_skips_on_overflow():
    """Three steps of the master pass on the head's weights from the gradient the call leaves, one of them overflowing: its
    flag makes the pass skip, and the weights stay as they were."""
    N, H, V = 128, 128, 2000
    c = Chain(N, H, V, 11, 1024.0)
    b = c.b
    w32 = c.Wd.float().reshape(-1).contiguous()
    flags = torch.zeros(2, dtype=torch.int32, device="cuda")
    for S, skipped in ((1024.0, False), (2.0 ** 26, True), (1024.0, False)):
        c.S = S
        before = w32.clone()
        flags.zero_()
        c.flag = flags[:1]
        c.run()
        b.mpt_update_flat(c.dW, w32, None, c.Wd, V * H, 1.0 / S, 0.5, 0.0, 0, 0, flags)
        torch.cuda.synchronize()
        assert bool((w32 == before).all()) == skipped
        if not skipped:
            expect = before - 0.5 * (c.dW.float().reshape(-1) * (1.0 / S))
            assert torch.equal(w32, expect) and torch.equal(c.Wd.reshape(-1), expect.half())


def test_two_chains_at_once_give_what_they_give_alone():
    """Two chains with buffers and workspaces of their own, on two streams, interleaved call by call, eager and as two captured
    graphs replayed side by side."""
    chains = [Chain(300, 512, 9000, 21, 2048.0), Chain(520, 264, 20000, 22, 4096.0)]
    alone = []
    for c in chains:
        c.run()
        torch.cuda.synchronize()
        alone.append(c.outputs())
    streams = [torch.cuda.Stream() for _ in chains]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for c, s in zip(chains, streams):
            with torch.cuda.stream(s):
                c.run()
    torch.cuda.synchronize()
    for c, ref in zip(chains, alone):
        assert all(torch.equal(a, r) for a, r in zip(c.outputs(), ref))
    graphs = []
    for c, s in zip(chains, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s):
            with torch.cuda.graph(g, stream=s):
                c.run()
        graphs.append(g)
    for c in chains:
        for o in (c.x, c.dx, c.dW, c.dh, c.dg, c.db):
            o.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for c, ref in zip(chains, alone):
        assert all(torch.equal(a, r) for a, r in zip(c.outputs(), ref))


FIRST_CALLS = """
import torch
from paper_1710_03740_b200 import binding as b
torch.manual_seed(5)
N, H, V, K, S = 300, 520, 20011, 12, 512.0
f16 = lambda *s: torch.randn(*s, device="cuda").half()
x, gamma, beta, W, t = f16(N, H), f16(H), f16(H), f16(V, H) * 0.05, f16(N, K)
z = f16(N, 20016)
y = torch.randint(0, V, (N,), device="cuda", dtype=torch.int32)
idx = torch.randint(0, V, (N, K), device="cuda", dtype=torch.int32)
h, dh, dx, dW, dz = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty_like(W), torch.empty_like(z)
dg, db = torch.empty_like(gamma), torch.empty_like(beta)
mean, rstd, rl, loss, rl2, loss2 = (torch.empty(n, device="cuda") for n in (N, N, N, 1, N, 1))
wn = torch.empty(b.mpt_layernorm_workspace_bytes(N, H), dtype=torch.uint8, device="cuda")
wl = torch.empty(b.mpt_linear_ce_workspace_bytes(N, V, H), dtype=torch.uint8, device="cuda")
status = torch.zeros(1, dtype=torch.int32, device="cuda")
outs = (h, dh, dx, dW, dz[:, :V], dg, db, mean, rstd, rl, loss, rl2, loss2)

def run():
    b.mpt_layernorm_forward(N, H, x, H, gamma, beta, 1e-5, h, H, mean, rstd, status)
    b.mpt_linear_ce(N, V, H, h, H, W, H, y, S, rl, loss, dh, H, dW, H, wl, status=status)
    b.mpt_layernorm_backward(N, H, dh, H, x, H, gamma, mean, rstd, dx, H, dg, db, wn, status=status)
    b.mpt_distill_topk(z, 20016, N, V, t, idx, K, K, 2.0, S, dz, 20016, rl2, loss2, status)

graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    run()
for o in outs:
    o.fill_(7.0)
graph.replay()
torch.cuda.synchronize()
replayed = [o.clone() for o in outs]
run()
torch.cuda.synchronize()
assert int(status) == 0
assert all(torch.equal(a, o) for a, o in zip(replayed, outs))
print("alike")
"""


def test_first_calls_of_a_process_are_captured():
    """What a call sets up once per process and device is allowed while a stream is captured."""
    import subprocess
    import sys
    from pathlib import Path
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], capture_output=True, text=True, timeout=300, cwd=Path(__file__).parents[1])
    assert r.returncode == 0 and "alike" in r.stdout, r.stderr[-2000:]
