"""The node-wise operators together, as a relational layer uses them: layer norm that leaves its rows in 8 bits, the transform by
type, and both backward passes from what was left; also replayed from a HIP graph, on other streams, and beside the aggregation."""
import numpy as np
import pytest
import torch

from paper_2111_06483_amd import sar
from tests import gpu_util as gu
from tests import nodewise as nw

pytestmark = pytest.mark.gpu
EPS = 1e-5


class Layer:
    def __init__(self, n, K, F, ends, dtype, seed=0):
        g = torch.Generator().manual_seed(seed)
        rn = lambda *s: torch.randn(*s, generator=g)
        self.n, self.K, self.F, self.ends, self.T, self.dtype = n, K, F, ends, len(ends) - 1, dtype
        self.X, self.dZ = rn(n, K).to(dtype).cuda(), rn(n, F).to(dtype).cuda()
        self.gamma, self.beta = (1 + 0.1 * rn(K)).cuda(), (0.1 * rn(K)).cuda()
        self.W = (rn(self.T, K, F) / K ** 0.5).cuda()
        self.ptr = torch.tensor(ends, dtype=torch.int32, device="cuda")
        e = lambda *s, dt=dtype: torch.zeros(*s, dtype=dt, device="cuda")
        f32 = torch.float32
        self.Y, self.Z, self.dY, self.dX = e(n, K), e(n, F), e(n, K), e(n, K)
        self.stats, self.dW, self.dg, self.db = e(n, 2, dt=f32), e(self.T, K, F, dt=f32), e(K, dt=f32), e(K, dt=f32)
        self.Xp, self.Yp = sar.packed_empty(n, K), sar.packed_empty(n, K)
        self.lwork = torch.empty(sar.sar_linear_typed_workspace_bytes(n, K, F, self.T), dtype=torch.uint8, device="cuda")
        self.nwork = torch.empty(sar.sar_layernorm_workspace_bytes(n, K), dtype=torch.uint8, device="cuda")

    def forward(self):
        sar.sar_layernorm_fwd(self.X, self.gamma, self.beta, EPS, self.Y, self.stats, self.Xp, self.Yp)
        sar.sar_linear_typed_fwd(self.Y, self.W, self.ptr, self.Z, self.lwork)

    def backward(self):
        sar.sar_linear_typed_bwd(self.Yp, self.dZ, self.W, self.ptr, False, self.dW, self.dY, self.lwork)
        sar.sar_layernorm_bwd(self.dY, self.Xp, self.stats, self.gamma, False, self.dX, self.dg, self.db, self.nwork)

    def step(self):
        self.forward()
        self.backward()

    def outputs(self):
        return [t.clone() for t in (self.Y, self.Z, self.stats, self.dW, self.dY, self.dX, self.dg, self.db, *self.Xp, *self.Yp)]


def close(got, want, rel):
    assert np.abs(nw.f64(got) - want).max() <= rel * np.abs(want).max()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,K,F,ends", [(700, 100, 47, [0, 300, 300, 690]), (30_000, 256, 256, [0, 10_000, 10_007, 30_000])])
def test_a_layer(n, K, F, ends, dtype):
    s = Layer(n, K, F, ends, dtype)
    s.step()
    # every call against 64 bits, on what it was given (the rows in 8 bits are what they stand for)
    x, g = nw.f64(s.X), nw.f64(s.gamma)
    xp = nw.unpack(s.Xp[0].cpu().numpy(), s.Xp[1].cpu().numpy(), K)
    yp = nw.unpack(s.Yp[0].cpu().numpy(), s.Yp[1].cpu().numpy(), K)
    y, mean, r = nw.norm_fwd(x, g, nw.f64(s.beta), EPS)
    # roundings of the stored type (half a step) and some tens of fp32 ones; sums of at most 256 terms, or n / 256 + 128
    rel = nw.HALF[dtype] + 300 * nw.U
    close(s.Y, y, rel)
    d, w, Yd = nw.f64(s.dZ), nw.f64(s.W), nw.f64(s.Y)
    Z, dY, dW = np.zeros((n, F)), np.zeros((n, K)), np.zeros_like(w)
    for t, lo, hi in nw.spans(ends, n):
        Z[lo:hi], dY[lo:hi], dW[t] = Yd[lo:hi] @ w[t], d[lo:hi] @ w[t].T, yp[lo:hi].T @ d[lo:hi]
    # (bf16: the weights' 16 bits too, a term's error of 2^-16 over up to 256 terms of one size)
    close(s.Z, Z, rel + (2.0 ** -12 if dtype == torch.bfloat16 else 0))
    close(s.dY, dY, rel + (2.0 ** -12 if dtype == torch.bfloat16 else 0))
    close(s.dW, dW, (64 + n / 32) * 2 * nw.U)
    st = nw.f64(s.stats)
    dx, dg, db = nw.norm_bwd(nw.f64(s.dY), xp, st[:, :1], st[:, 1:], g)
    close(s.dX, dx, rel)
    close(s.dg, dg, (128 + n / 256) * nw.U * np.sqrt(n))
    close(s.db, db, (128 + n / 256) * nw.U * np.sqrt(n))
    # and the whole against the layer without 8 bits: a value is off by at most 2^-7 of its block's largest, errors of either sign
    full = np.zeros_like(w)
    for t, lo, hi in nw.spans(ends, n):
        full[t] = y[lo:hi].T @ d[lo:hi]
    dxf, dgf, _ = nw.norm_bwd(dY, x, mean, r, g)
    norm = np.linalg.norm
    for got, want in ((s.dW, full), (s.dX, dxf), (s.dg, dgf)):
        assert norm(nw.f64(got) - want) <= (2.0 ** -6 + 2 * nw.HALF[dtype]) * norm(want)


@pytest.mark.parametrize("n,K,F", [(500, 96, 64), (5000, 200, 70), (70_000, 128, 256)])
def test_a_replayed_graph_and_an_eager_layer_beside_it(n, K, F):
    """Two layers recorded into one graph share their scratch, one after the other; between the replays the same calls run eagerly."""
    a, b = (Layer(n, K, F, [0, n // 3, n // 3, n - 10], dt, seed=k) for k, dt in enumerate([torch.float32, torch.bfloat16]))
    size = max(a.lwork.numel(), b.lwork.numel())
    a.lwork = b.lwork = torch.empty(size, dtype=torch.uint8, device="cuda")
    a.step(), b.step()                                           # (a first call of each kernel outside the recording)
    want = [a.outputs(), b.outputs()]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            a.step()
            b.step()
    for _ in range(3):
        for layer in (a, b):
            for t in (layer.Y, layer.Z, layer.dW, layer.dX, layer.dg, layer.Xp[0], layer.Yp[1]):
                t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for layer, w in zip((a, b), want) for x, y in zip(layer.outputs(), w))
        b.step(), a.step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for layer, w in zip((a, b), want) for x, y in zip(layer.outputs(), w))


def test_the_current_stream_is_the_one():
    """Work goes to the stream that is current: behind what another call on it still has to write."""
    s = Layer(20_000, 128, 128, [0, 9000, 20_000], torch.float32)
    s.step()
    want = s.outputs()
    x = s.X.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.X.zero_()
        for _ in range(20):
            s.X.add_(x, alpha=0.0)                               # (something to wait for)
        s.X.copy_(x)
        s.step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(s.outputs(), want))


def test_before_an_aggregation():
    """A relational layer: norm, transform by type, mean over the neighbours, and back."""
    from tests.helpers import rel_err, tiny_graph
    rng = np.random.default_rng(11)
    N, K, F = 240, 40, 24
    src, dst, part = tiny_graph(rng, N, 2400, 1)
    ends = [0, 100, 100, 240]
    s = Layer(N, K, F, ends, torch.float32, seed=3)
    b = gu.build_blocks(src, dst, part, 1, 0)
    s.forward()
    out = torch.empty(N, F, device="cuda")
    sar.sar_spmm_all(b, [s.Z], True, out)
    G = torch.randn(N, F, generator=torch.Generator().manual_seed(8)).cuda()
    sar.sar_spmm_bwd_all(b, G, True, [s.dZ])
    s.backward()
    deg = np.maximum(np.bincount(dst, minlength=N), 1)[:, None]
    y, mean, r = nw.norm_fwd(nw.f64(s.X), nw.f64(s.gamma), nw.f64(s.beta), EPS)
    w = nw.f64(s.W)
    Z = np.concatenate([y[lo:hi] @ w[t] for t, lo, hi in nw.spans(ends, N)])
    want = np.zeros((N, F))
    np.add.at(want, dst, Z[src])
    assert rel_err(nw.f64(out), want / deg) < 1e-5               # (a hundred fp32 roundings of terms of one size)
    dZ = np.zeros((N, F))
    np.add.at(dZ, src, (nw.f64(G) / deg)[dst])
    dY = np.concatenate([dZ[lo:hi] @ w[t].T for t, lo, hi in nw.spans(ends, N)])
    assert rel_err(nw.f64(s.dY), dY) < 1e-5
    dx, dg, _ = nw.norm_bwd(dY, nw.f64(s.X), mean, r, nw.f64(s.gamma))
    assert np.linalg.norm(nw.f64(s.dX) - dx) < 2.0 ** -6 * np.linalg.norm(dx)     # (from 8 bits)
    assert np.linalg.norm(nw.f64(s.dg) - dg) < 2.0 ** -6 * np.linalg.norm(dg)
    b.close()


def test_tensors_on_the_device_that_do_not_fit():
    s = Layer(10, 16, 8, [0, 5, 10], torch.float32)
    with pytest.raises(sar.SarError, match="host memory"):
        sar.sar_layernorm_fwd(s.X, s.gamma.cpu(), s.beta, EPS, s.Y)
    with pytest.raises(sar.SarError, match="host memory"):
        sar.sar_pack(s.X, (s.Xp[0], s.Xp[1].cpu()))
    with pytest.raises(sar.SarError, match="needs"):
        sar.sar_linear_typed_fwd(s.Y, s.W, s.ptr, s.Z, s.lwork[:16])
    with pytest.raises(sar.SarError, match="alias"):
        sar.sar_linear_typed_bwd(s.X, s.X, torch.zeros(2, 16, 16, device="cuda"), s.ptr, False, None, s.X,
                                 torch.empty(sar.sar_linear_typed_workspace_bytes(10, 16, 16, 2), dtype=torch.uint8, device="cuda"))
