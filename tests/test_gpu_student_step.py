"""The transform with its epilogue, log probabilities and distillation together, as a student network is taught: two layers, the loss against a teacher's top
classes and the labels, and the gradients; also replayed from HIP graphs, on other streams, at any address and beyond 2^31 values."""
import numpy as np
import pytest
import torch

from paper_2111_06483_amd import sar
from tests import classrows as cr
from tests import nodewise as nw
from tests.test_gpu_class_rows import check_results
from tests.test_gpu_linear_act import act

pytestmark = pytest.mark.gpu
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32
DTYPES = [F32, BF16]
T = 2.0


def bytes_of(size):
    return torch.empty(size, dtype=torch.uint8, device="cuda")


class Student:
    """X -> gelu(X W1 + b1) + R -> logits; teacher logits [n, C] of its own; half of the loss from each."""

    def __init__(self, n, K, F, C, dtype, k=5, seed=0):
        g = torch.Generator().manual_seed(seed)
        rn = lambda *s, dt=F32: torch.randn(*s, generator=g).to(dt).cuda()
        e = lambda *s, dt=F32: torch.zeros(*s, dtype=dt, device="cuda")
        self.n, self.K, self.F, self.C, self.k, self.dtype = n, K, F, C, k, dtype
        self.X, self.R, self.teacher = rn(n, K, dt=dtype), rn(n, F, dt=dtype), (3 * rn(n, C)).to(dtype)
        self.W1, self.b1, self.W2, self.b2 = rn(K, F) / K ** 0.5, rn(F), rn(F, C) / F ** 0.5, rn(C)
        self.label = torch.randint(-1, C, (n,), generator=g, dtype=I32).cuda()
        self.top = (e(n, k), e(n, k, dt=I32))
        self.H, self.A1, self.Z = e(n, F, dt=dtype), e(n, F, dt=dtype), e(n, C, dt=dtype)
        self.loss, self.lse, self.lseT, self.logp, self.entropy = (e(n) for _ in range(5))
        self.minus, self.half = torch.full((n,), -0.5, device="cuda"), torch.full((n,), 0.5, device="cuda")
        self.dZ, self.dZ2, self.dH, self.dX = e(n, C, dt=dtype), e(n, C, dt=dtype), e(n, F, dt=dtype), e(n, K, dt=dtype)
        self.dW1, self.db1, self.dW2, self.db2 = e(K, F), e(F), e(F, C), e(C)
        self.work = bytes_of(max(sar.sar_linear_act_workspace_bytes(n, K, F), sar.sar_linear_act_workspace_bytes(n, F, C),
                                 sar.sar_logprob_workspace_bytes(n, C, k), sar.sar_distill_workspace_bytes(n, C, k)))

    def step(self):
        sar.sar_logprob_fwd(self.teacher, None, None, None, None, self.top, self.work)
        sar.sar_linear_act_fwd(self.X, self.W1, self.b1, self.R, sar.SAR_ACT_GELU, True, self.H, self.A1, self.work)
        sar.sar_linear_act_fwd(self.H, self.W2, self.b2, None, sar.SAR_ACT_NONE, False, self.Z, None, self.work)
        sar.sar_logprob_fwd(self.Z, self.label, self.logp, self.lse, self.entropy, None, self.work)
        sar.sar_distill_fwd(self.Z, self.top, T, self.loss, self.lseT, self.work)
        sar.sar_logprob_bwd(self.Z, self.label, self.lse, None, self.minus, None, self.dZ2)
        sar.sar_distill_bwd(self.Z, self.top, T, self.lseT, self.half, self.dZ)
        self.dZ += self.dZ2
        sar.sar_linear_act_bwd(self.dZ, None, self.H, self.W2, sar.SAR_ACT_NONE, False, self.dW2, self.db2, self.dH, None, self.work)
        sar.sar_linear_act_bwd(self.dH, self.A1, self.X, self.W1, sar.SAR_ACT_GELU, False, self.dW1, self.db1, self.dX, None, self.work)

    def outputs(self):
        return [t.clone() for t in (*self.top, self.H, self.A1, self.Z, self.logp, self.entropy, self.loss, self.dZ, self.dW2, self.db2, self.dH, self.dW1, self.db1,
                                    self.dX)]


def near(got, want, rel):
    size = np.abs(want).max()
    assert np.abs(nw.f64(got) - want).max() <= rel * size + 1e-30


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,K,F,C", [(300, 40, 64, 47), (9000, 100, 128, 172), (300, 16, 24, 5000), (70_000, 100, 64, 47)])
def test_a_step(n, K, F, C, dtype):
    s = Student(n, K, F, C, dtype)
    s.step()
    # every call against 64 bits, on what it was given; rounding of the stored type, and fp32 sums' (of up to 5000 terms, rows' sums n / 256 + 64)
    rel = nw.HALF[dtype] + (300 + n / 256) * 2 * nw.U + (2.0 ** -12 if dtype == BF16 else 0)
    x, h, z = nw.f64(s.X), nw.f64(s.H), nw.f64(s.Z)
    assert (s.top[1].cpu().numpy() == cr.top(nw.f64(s.teacher), s.k)).all()
    a = x @ nw.f64(s.W1) + nw.f64(s.b1)
    near(s.A1, a, rel)
    gelu = [v.cpu().numpy() for v in act("gelu", torch.from_numpy(a))]
    near(s.H, gelu[0] + nw.f64(s.R), rel)
    near(s.Z, h @ nw.f64(s.W2) + nw.f64(s.b2), rel)
    label, value, index = s.label.cpu().numpy(), nw.f64(s.top[0]), s.top[1].cpu().numpy()
    soft = cr.Softmax(z)
    own = np.where(label >= 0, soft.logp[np.arange(n), np.maximum(label, 0)], 0.0)
    near(s.logp, own, rel)
    near(s.entropy, soft.entropy[:, 0], rel)
    near(s.loss, cr.distill_fwd(z, value, index, T)[0], rel)
    d = (cr.distill_bwd(z, value, index, T, cr.Softmax(z, T).lse[:, 0], np.full(n, 0.5))[0] +
         cr.logprob_bwd(z, soft.lse[:, 0], soft.entropy[:, 0], label, np.full(n, -0.5), np.zeros(n))[0])
    near(s.dZ, d, 3 * rel)
    d = nw.f64(s.dZ)
    near(s.dW2, h.T @ d, rel)
    near(s.db2, d.sum(0), rel)
    near(s.dH, d @ nw.f64(s.W2).T, rel)
    d = nw.f64(s.dH) * act("gelu", torch.from_numpy(nw.f64(s.A1)))[1].numpy()
    near(s.dW1, x.T @ d, rel + 2.0 ** -16)
    near(s.db1, d.sum(0), rel)
    near(s.dX, d @ nw.f64(s.W1).T, 2 * rel)


SIZES = [(500, 40, 64, 47), (20_000, 100, 64, 172), (70_000, 64, 128, 47), (40, 16, 24, 20_000)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,K,F,C", SIZES)
def test_the_same_bits_every_time(n, K, F, C, dtype):
    s = Student(n, K, F, C, dtype, seed=1)
    s.step()
    first = s.outputs()
    s.work.fill_(0xff)                                     # (nothing of a call is left for the next one)
    s.step()
    assert all(torch.equal(a, b) for a, b in zip(first, s.outputs()))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,K,F,C", SIZES)
def test_replayed_from_graphs(n, K, F, C, dtype):
    """Two captured steps with scratch of their own, replayed in turn with new inputs and eager work between the replays."""
    students = [Student(n, K, F, C, dtype, seed=k) for k in (2, 3)]
    graphs = []
    side = torch.cuda.Stream()
    for s in students:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            s.step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.step()
        graphs.append(g)
    other = Student(n, K, F, C, dtype, seed=4)
    for turn in range(3):
        for s, g in zip(students, graphs):
            s.X.copy_(torch.randn(n, K, generator=torch.Generator().manual_seed(turn)).to(dtype))
            s.teacher.mul_(0.9)
            for t in (s.H, s.Z, s.loss, s.dZ, s.dW1, s.db1, s.dW2, s.dX):
                t.zero_()
            g.replay()
            other.step()
            torch.cuda.synchronize()
            got = s.outputs()
            s.step()
            assert all(torch.equal(a, b) for a, b in zip(got, s.outputs())), turn


@pytest.mark.parametrize("dtype", DTYPES)
def test_two_streams_at_once(dtype):
    n, K, F, C = 70_000, 64, 128, 172
    students = [Student(n, K, F, C, dtype, seed=k) for k in (5, 6)]
    want = []
    for s in students:
        s.step()
        want.append(s.outputs())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in students]
    for _ in range(4):
        for s, st in zip(students, streams):
            with torch.cuda.stream(st):
                s.step()
    torch.cuda.synchronize()
    for s, w in zip(students, want):
        assert all(torch.equal(a, b) for a, b in zip(s.outputs(), w))


def moved(t, by):
    """The same values, `by` elements behind a boundary of 256 bytes, with room behind that must stay as it is."""
    room = torch.full((t.numel() + by + 64,), 77, dtype=t.dtype, device="cuda")
    v = room[by:by + t.numel()].view(t.shape)
    v.copy_(t)
    return v, room


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("by", [1, 3])
@pytest.mark.parametrize("n,K,F,C", [(301, 33, 47, 47), (66_000, 47, 70, 9), (66_001, 47, 72, 100), (20, 17, 64, 5001)])
def test_tensors_at_any_address(n, K, F, C, by, dtype):
    s = Student(n, K, F, C, dtype, seed=7)
    s.step()
    want = s.outputs()
    names = ["X", "R", "teacher", "W1", "b1", "W2", "b2", "label", "H", "A1", "Z", "loss", "lse", "lseT", "logp", "entropy", "minus", "half", "dZ", "dZ2", "dH", "dX", "dW1",
             "db1", "dW2", "db2"]
    rooms = []
    for name in names:
        v, room = moved(getattr(s, name), by)
        setattr(s, name, v)
        rooms.append((name, room, v.numel()))
    tops = [moved(t, by) for t in s.top]
    s.top = tuple(v for v, _ in tops)
    rooms += [("top", room, v.numel()) for v, room in tops]
    s.step()
    assert all(torch.equal(a, b) for a, b in zip(want, s.outputs()))
    for name, room, count in rooms:
        assert bool((room[:by] == 77).all()) and bool((room[by + count:] == 77).all()), name


def test_rows_beyond_two_to_the_31_values():
    """The last rows, in 64 bits."""
    n, C, k, tail = 12_600_000, 172, 3, 4096
    X = torch.randn(1 << 20, C, dtype=BF16, device="cuda").repeat(13, 1)[:n].contiguous()
    label = torch.randint(-1, C, (n,), dtype=I32, device="cuda")
    e = lambda *s, dt=F32: torch.empty(n, *s, dtype=dt, device="cuda")
    logp, lse, H, top, loss, lseT, one, dX = e(), e(), e(), (e(k), e(k, dt=I32)), e(), e(), torch.ones(n, device="cuda"), torch.empty_like(X)
    sar.sar_logprob_fwd(X, label, logp, lse, H, top)
    last = slice(n - tail, n)
    check_results(X[last], label[last], k, logp[last], lse[last], H[last], tuple(t[last] for t in top))
    sar.sar_distill_fwd(X, top, T, loss, lseT)
    x, v, c, g = cr.f64(X[last]), cr.f64(top[0][last]), top[1][last].cpu().numpy(), np.ones(tail)
    want, off, s = cr.distill_fwd(x, v, c, T)
    assert (np.abs(cr.f64(loss[last]) - want) <= off).all() and (np.abs(cr.f64(lseT[last]) - s.lse[:, 0]) <= s.off_lse[:, 0]).all()

    def check(want, off):
        assert (np.abs(cr.f64(dX[last]) - want) <= off + cr.half_step(BF16)(np.abs(want) + off)).all()
    sar.sar_logprob_bwd(X, label, lse, H, one, one, dX)
    check(*cr.logprob_bwd(x, cr.f64(lse[last]), cr.f64(H[last]), label[last].cpu().numpy(), g, g))
    sar.sar_distill_bwd(X, top, T, lseT, one, dX)
    check(*cr.distill_bwd(x, v, c, T, cr.f64(lseT[last]), g))


def test_the_transform_beyond_two_to_the_31_values():
    n, K, F, tail = 8_500_000, 256, 256, 4096
    X = torch.randn(1 << 20, K, dtype=BF16, device="cuda").repeat(9, 1)[:n].contiguous()
    W, b = torch.randn(K, F, device="cuda") / 16, torch.randn(F, device="cuda")

    def run(X):
        m = X.shape[0]
        Y, A, dX = torch.empty(m, F, dtype=BF16, device="cuda"), torch.empty(m, F, dtype=BF16, device="cuda"), torch.empty_like(X)
        work = bytes_of(sar.sar_linear_act_workspace_bytes(m, K, F))
        sar.sar_linear_act_fwd(X, W, b, X, sar.SAR_ACT_SILU, True, Y, A, work)
        sar.sar_linear_act_bwd(Y, A, None, W, sar.SAR_ACT_SILU, False, None, None, dX, None, work)
        return [t[-tail:].clone() for t in (Y, A, dX)]
    whole, alone = run(X), run(X[-tail - 102_400:].contiguous())
    assert all(torch.equal(a, b) for a, b in zip(whole, alone))
