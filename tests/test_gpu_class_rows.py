"""Log probabilities, entropy and top classes of rows of scores, distillation from a teacher's top classes, and their gradients, against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2111_06483_amd import sar
from tests import classrows as cr

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DTYPES = [F32, BF16]
# every number of lanes and pieces of a row, on both sides of each line, whole and ragged; long rows in one part and in several
CLASSES = [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 47, 64, 65, 96, 97, 100, 127, 128, 129, 172, 192, 193, 255, 256, 257, 384, 500, 512, 513, 777, 1000,
           1024, 1025, 1536, 2047, 2048, 2049, 3000, 4095, 4096, 4097, 5001, 8191, 8193, 16385, 20_001, 65_536]


def scores(n, C, dtype, seed=0):
    g = torch.Generator().manual_seed(seed * 7919 + n * 31 + C)
    x = torch.randn(n, C, generator=g) * (0.5 + 3 * torch.rand(n, 1, generator=g)) + 4 * torch.randn(n, 1, generator=g)
    label = torch.randint(0, C, (n,), generator=g, dtype=torch.int32)
    label[torch.rand(n, generator=g) < 0.3] = -1
    return x.to(dtype).cuda(), label.cuda()


def scratch(size):
    """Scratch of exactly that size, and what lies behind it."""
    room = torch.full((size + 256,), 77, dtype=torch.uint8, device="cuda")
    return (room[:size] if size else None), room[size:]


def forward(X, label, k):
    n, C = X.shape
    e = lambda *s, dt=F32: torch.full(s, -7, dtype=dt, device="cuda")
    logp, lse, entropy, top = e(n), e(n), e(n), (e(n, k), e(n, k, dt=torch.int32))
    work, behind = scratch(sar.sar_logprob_workspace_bytes(n, C, k))
    sar.sar_logprob_fwd(X, label, logp, lse, entropy, top, work)
    assert bool((behind == 77).all())
    return logp, lse, entropy, top


def check_forward(X, label, k):
    check_results(X, label, k, *forward(X, label, k))


def check_results(X, label, k, logp, lse, entropy, top):
    n, C = X.shape
    logp, lse, entropy = cr.f64(logp), cr.f64(lse), cr.f64(entropy)
    x, lab = cr.f64(X), label.cpu().numpy()
    some = ~np.isneginf(x).all(1)
    assert np.isneginf(lse[~some]).all() and (entropy[~some] == 0).all() and np.isneginf(logp[~some & (lab >= 0) & (lab < C)]).all()
    assert np.isneginf(cr.f64(top[0])[~some]).all() and (top[1].cpu().numpy()[~some] == -1).all()
    x, lab, logp, lse, entropy = x[some], lab[some], logp[some], lse[some], entropy[some]
    s = cr.Softmax(x)
    assert (np.abs(lse - s.lse[:, 0]) <= s.off_lse[:, 0]).all()
    assert (np.abs(entropy - s.entropy[:, 0]) <= s.off_entropy[:, 0]).all()
    has = (lab >= 0) & (lab < C)
    rows, at = np.nonzero(has)[0], lab[has]
    assert (logp[~has] == 0).all()
    want = s.logp[rows, at]
    masked = np.isneginf(want)
    assert np.isneginf(logp[has][masked]).all()
    with np.errstate(all="ignore"):
        near = np.abs(logp[has] - want) <= s.off_log[rows, 0] + 3 * cr.U * (np.abs(s.d[rows, at]) + np.abs(want))
    assert near[~masked].all()
    value, index = cr.f64(top[0])[some], top[1].cpu().numpy()[some]
    want = cr.top(x, k)
    assert (index == want).all()
    none, at = want < 0, np.where(want < 0, 0, want)
    assert np.isneginf(value[none]).all()
    d, v = np.take_along_axis(s.d, at, 1), np.take_along_axis(s.logp, at, 1)
    assert (np.abs(value - v) <= s.off_logp(d, v))[~none].all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", CLASSES)
def test_forward_of_every_width(C, dtype):
    n = 301 if C <= 600 else 37 if C <= 5001 else 5
    X, label = scores(n, C, dtype)
    check_forward(X, label, 5)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,C,k", [(1, 47, 8), (3, 47, 47), (5, 10, 64), (2, 172, 64), (700, 172, 8), (70_001, 47, 1), (9, 300, 33), (1, 2048, 64), (4, 3000, 64),
                                   (1, 131_075, 64), (64, 65_536, 8), (1023, 9000, 3), (1025, 4100, 2), (2, 700_001, 17)])
def test_top_classes(n, C, k, dtype):
    X, label = scores(n, C, dtype, 1)
    check_forward(X, label, k)


@pytest.mark.parametrize("n,C,k", [(270_001, 172, 8), (262_147, 129, 3), (262_145, 190, 20), (131_075, 301, 8), (65_537, 577, 2)])
def test_many_rows_of_bf16(n, C, k):
    """More values a lane where there are many rows: 701 rows over and over, each as its first one is."""
    few = 701
    base, label = scores(few, C, BF16, 17)
    base[5], base[9, : C - 1] = float("-inf"), float("-inf")
    turn = torch.arange(n, device="cuda") % few
    logp, lse, entropy, (value, index) = forward(base[turn], label[turn], k)
    first = slice(0, few)
    check_results(base, label, k, logp[first], lse[first], entropy[first], (value[first], index[first]))
    for t in (logp, lse, entropy, value, index):
        assert torch.equal(t, t[first][turn])
    top = teacher(few, C, min(k, 4), 4)
    want, off, s = cr.distill_fwd(cr.f64(base), cr.f64(top[0]), top[1].cpu().numpy(), 2.0)
    loss, lse = torch.full((n,), -7.0, device="cuda"), torch.full((n,), -7.0, device="cuda")
    sar.sar_distill_fwd(base[turn], tuple(t[turn] for t in top), 2.0, loss, lse)
    some = np.isfinite(want)       # (otherwise the student has no score for a listed class, or none at all: an infinite loss)
    assert (np.abs(cr.f64(loss[first]) - want)[some] <= off[some]).all() and np.isposinf(cr.f64(loss[first])[~some]).all()
    for t in (loss, lse):
        assert torch.equal(t, t[first][turn])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("k", [0, 1, 3, 4, 6, 7])
@pytest.mark.parametrize("C", [1, 2, 3, 4, 5, 7, 8, 9, 12, 16])
def test_few_classes(C, k, dtype):
    """A row by one lane, two or four; the last rows' pieces pass the tensor's end."""
    for n in (1, 2, 256, 1025):
        X, label = scores(n, C, dtype, 15)
        X[n // 2] = float("-inf")
        check_forward(X, label, k)
    check_distill(scores(1025, C, dtype, 16)[0], teacher(1025, C, k, 3), 1.5, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,C,k", [(511, 8193, 2), (512, 8193, 2), (300, 9000, 5), (255, 9000, 64), (40, 20_000, 64), (3, 1_000_003, 8), (1, 300_001, 64), (6, 262_144, 0)])
def test_rows_in_parts(n, C, k, dtype):
    """A row by one workgroup, by a few, by the most there are; rows whose top classes are in one part, and in every part as many."""
    X, label = scores(n, C, dtype, 14)
    for row, x in ((1, torch.linspace(-8, 8, C)), (2, torch.linspace(8, -8, C)), (3, (torch.arange(C) % 4096 == 77) * 4.0)):
        if row < n:
            X[row] = x.to(dtype)
    check_forward(X, label, k)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", [6, 47, 172, 1001, 3001, 30_001])
def test_equal_scores(C, dtype):
    """Of few different values, -0 and 0 among them; rows of one value; rising and falling rows."""
    n = 12
    g = torch.Generator().manual_seed(C)
    x = torch.randint(-1, 2, (n, C), generator=g).float()
    x[x == 0] = torch.where(torch.rand(int((x == 0).sum()), generator=g) < 0.5, -0.0, 0.0)
    x[1] = 3.0
    x[2], x[3] = torch.linspace(-8, 8, C), torch.linspace(8, -8, C)
    x[4] = -2.5
    X = x.to(dtype).cuda()
    check_forward(X, torch.arange(n, dtype=torch.int32).clamp(max=C - 1).cuda(), min(C, 64))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", [5, 47, 172, 900, 2500, 20_000])
def test_masked_classes(C, dtype):
    """Scores of -inf, rows that keep one class or none, the type's lowest number as a mask, a label that is masked."""
    n = 10
    X, label = scores(n, C, dtype, 3)
    label = label.clamp(min=0)
    g = torch.Generator().manual_seed(5)
    X[(torch.rand(n, C, generator=g) < 0.5).cuda()] = -float("inf")
    X[:, 0] = 1.5                                              # (a class that every row has)
    X[0] = -float("inf")
    X[1] = -float("inf")
    X[1, C - 1] = 2.0
    X[2] = torch.finfo(dtype).min
    X[2, 1] = -1.0
    X[3] = torch.finfo(dtype).min
    label[4] = C - 1
    X[4, C - 1] = -float("inf")
    k = min(C, 8)
    logp, lse, entropy, top = forward(X, label, k)
    inf = float("inf")
    assert lse[0] == -inf and entropy[0] == 0 and logp[0] == -inf and (top[1][0] == -1).all() and (top[0][0] == -inf).all()
    assert lse[1] == 2.0 and entropy[1] == 0 and top[1][1].tolist() == [C - 1] + [-1] * (k - 1) and top[0][1, 0] == 0
    assert lse[2] == -1 and entropy[2] == 0 and top[1][2].tolist()[:3] == [1, 0, 2][:k]
    assert abs(entropy[3].item() - np.log(C)) < 1e-5 and top[1][3].tolist() == list(range(k))
    assert logp[4] == -inf
    # the others as ever; -inf where the formula has it
    keep = [1, 5, 6, 7, 8, 9]
    x = cr.f64(X)[keep]
    s = cr.Softmax(x)
    assert (np.abs(cr.f64(lse)[keep] - s.lse[:, 0]) <= s.off_lse[:, 0]).all()
    assert (np.abs(cr.f64(entropy)[keep] - s.entropy[:, 0]) <= s.off_entropy[:, 0]).all()
    assert (top[1].cpu().numpy()[keep] == cr.top(x, k)).all()
    # gradients: nothing for a masked class, nothing in a row without classes
    dX, h = torch.full_like(X, 7), torch.ones(n, device="cuda")
    sar.sar_logprob_bwd(X, label, lse, entropy, h, h, dX)
    d = cr.f64(dX)
    own = np.arange(C)[None] == label.cpu().numpy()[:, None]
    assert np.isfinite(d).all() and (d[0] == 0).all() and (d[2][2:] == own[2][2:]).all()
    # (row 1's one class has all of the probability; its label may be a masked one, which is then pulled at by its weight, as in row 2)
    assert (d[1] == own[1] * 1.0 - (np.arange(C) == C - 1)).all()
    assert (d[np.isneginf(cr.f64(X)) & ~own] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", [5, 47, 900, 20_000])
def test_scores_that_are_no_numbers(C, dtype):
    """A NaN or an infinity spoils its own row's results and no other's."""
    n = 6
    X, label = scores(n, C, dtype, 4)
    label = label.clamp(min=0)
    clean = forward(X, label, min(C, 5))
    X[1, C // 2] = float("nan")
    X[3, 0] = float("inf")
    X[4] = float("nan")
    got = forward(X, label, min(C, 5))
    for a, b in zip(clean[:3], got[:3]):
        assert torch.isnan(b[[1, 3, 4]]).all() and torch.equal(a[[0, 2, 5]], b[[0, 2, 5]])
    i = got[3][1]
    assert torch.equal(clean[3][1][[0, 2, 5]], i[[0, 2, 5]]) and bool(((i >= -1) & (i < C)).all())
    one, dX = torch.ones(n, device="cuda"), torch.empty_like(X)
    sar.sar_logprob_bwd(X, label, got[1], got[2], one, one, dX)
    assert torch.isnan(dX[[1, 3, 4]].float()).all() and torch.isfinite(dX[[0, 2, 5]].float()).all()


def gradient_inputs(n, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(n, generator=g).cuda(), torch.randn(n, generator=g).cuda()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", CLASSES)
def test_backward_of_every_width(C, dtype):
    n = 701 if C <= 600 else 37 if C <= 5001 else 5
    X, label = scores(n, C, dtype, 6)
    label[::7] = C + 3                                      # (no class either)
    g, h = gradient_inputs(n, C)
    _, lse, entropy, _ = forward(X, label, 0)
    x, lab = cr.f64(X), label.cpu().numpy()
    for dl, dh in ((g, h), (g, None), (None, h)):
        dX = torch.full_like(X, 7)
        sar.sar_logprob_bwd(X, label if dl is not None else None, lse, entropy if dh is not None else None, dl, dh, dX)
        zero = np.zeros(n)
        want, off = cr.logprob_bwd(x, cr.f64(lse), cr.f64(entropy), lab, cr.f64(dl) if dl is not None else zero, cr.f64(dh) if dh is not None else zero)
        tol = off + (cr.half_step(dtype)(np.abs(want) + off) if dtype == BF16 else 0)
        assert (np.abs(cr.f64(dX) - want) <= tol).all()
    # in place
    dX2 = X.clone()
    sar.sar_logprob_bwd(dX2, None, lse, entropy, None, h, dX2)
    assert torch.equal(dX2, dX)


def test_gradients_by_differences():
    """Of the sum of the outputs by weights, in steps of a score (fp32; central differences of the formula in 64 bits)."""
    n, C = 4, 11
    X, label = scores(n, C, F32, 8)
    label = torch.tensor([3, -1, 0, 10], dtype=torch.int32, device="cuda")
    g, h = gradient_inputs(n, 3)
    _, lse, entropy, _ = forward(X, label, 0)
    dX = torch.empty_like(X)
    sar.sar_logprob_bwd(X, label, lse, entropy, g, h, dX)
    x, lab = cr.f64(X), label.cpu().numpy()

    def total(x):
        s = cr.Softmax(x)
        own = np.where(lab >= 0, s.logp[np.arange(n), np.maximum(lab, 0)], 0.0)
        return (cr.f64(g) * own + cr.f64(h) * s.entropy[:, 0]).sum()
    step = 1e-5
    for i in range(n):
        for c in range(C):
            up, down = x.copy(), x.copy()
            up[i, c] += step
            down[i, c] -= step
            # (a difference's own error: step^2 / 6 of the third derivative, some tens here; 2^-52 of the total over the step)
            assert abs((total(up) - total(down)) / (2 * step) - dX[i, c].item()) < 1e-6 + 64 * cr.U * (1 + abs(dX[i, c].item()) + np.abs(x).max())


# ---- distillation

def teacher(n, C, k, seed):
    """Lists with padding, a class named twice, rows without a class, a value of -inf."""
    g = torch.Generator().manual_seed(seed * 31 + C)
    value, index = 3 * torch.randn(n, k, generator=g), torch.randint(0, C, (n, k), generator=g, dtype=torch.int32)
    index[torch.rand(n, k, generator=g) < 0.1] = -1
    if k > 1:
        index[::3, 1] = index[::3, 0]
        index[1::4, k - 1] = C + 2
        value[2::5, 0] = -float("inf")
    if n > 2:
        index[n // 2] = -1
    return value.cuda(), index.cuda()


def check_distill(X, top, T, dtype):
    n, C = X.shape
    loss, lse = torch.full((n,), -7.0, device="cuda"), torch.full((n,), -7.0, device="cuda")
    work, behind = scratch(sar.sar_distill_workspace_bytes(n, C, top[0].shape[1]))
    sar.sar_distill_fwd(X, top, T, loss, lse, work)
    assert bool((behind == 77).all())
    x, v, i = cr.f64(X), cr.f64(top[0]), top[1].cpu().numpy()
    want, off, s = cr.distill_fwd(x, v, i, T)
    assert (np.abs(cr.f64(lse) - s.lse[:, 0]) <= s.off_lse[:, 0]).all()
    assert (np.abs(cr.f64(loss) - want) <= off).all()
    g, _ = gradient_inputs(n, C)
    dX = torch.full_like(X, 7)
    sar.sar_distill_bwd(X, top, T, lse, g, dX)
    want, off = cr.distill_bwd(x, v, i, T, cr.f64(lse), cr.f64(g))
    tol = off + (cr.half_step(dtype)(np.abs(want) + off) if dtype == BF16 else 0)
    assert (np.abs(cr.f64(dX) - want) <= tol).all()
    same = X.clone()
    sar.sar_distill_bwd(same, top, T, lse, g, same)
    assert torch.equal(same, dX)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", CLASSES)
def test_distillation_of_every_width(C, dtype):
    n = 701 if C <= 600 else 37 if C <= 5001 else 5
    X, _ = scores(n, C, dtype, 9)
    check_distill(X, teacher(n, C, 8, 1), 2.0, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,C,k,T", [(1, 1, 1, 1.0), (1, 47, 1, 0.7), (5, 47, 64, 3.0), (300, 47, 33, 1.0), (3, 5000, 64, 4.0), (2, 131_075, 64, 1.5), (40_001, 47, 3, 2.0),
                                     (4, 64, 0, 1.0), (64, 20_000, 16, 2.0)])
def test_lists_of_every_length(n, C, k, T, dtype):
    X, _ = scores(n, C, dtype, 10)
    check_distill(X, teacher(n, C, k, 2), T, dtype)


def test_a_teacher_that_is_the_student():
    """All classes listed with the student's own scores: no loss, no gradient (fp32 roundings)."""
    X, _ = scores(50, 47, F32, 11)
    lse, loss, logp = (torch.empty(50, device="cuda") for _ in range(3))
    top = (torch.empty(50, 47, device="cuda"), torch.empty(50, 47, dtype=torch.int32, device="cuda"))
    sar.sar_logprob_fwd(X, None, None, None, None, top)
    sar.sar_distill_fwd(X, top, 1.7, loss, lse)
    dX = torch.empty_like(X)
    sar.sar_distill_bwd(X, top, 1.7, lse, torch.ones(50, device="cuda"), dX)
    off = 300 * cr.U * (1 + X.abs().max().item())
    assert loss.abs().max() < off and dX.abs().max() < off


def test_distillation_of_masked_rows():
    X, _ = scores(5, 47, F32, 12)
    inf = float("inf")
    X[0] = -inf                                             # no class
    X[1, 3] = -inf                                          # one that the teacher has
    X[2, 40:] = -inf
    X[3, 5] = float("nan")
    value, index = torch.randn(5, 4).cuda(), torch.tensor([[3, 7, 9, 12]] * 5, dtype=torch.int32, device="cuda")
    loss, lse, dX = torch.empty(5, device="cuda"), torch.empty(5, device="cuda"), torch.empty_like(X)
    sar.sar_distill_fwd(X, (value, index), 2.0, loss, lse)
    sar.sar_distill_bwd(X, (value, index), 2.0, lse, torch.ones(5, device="cuda"), dX)
    assert loss[0] == inf and (dX[0] == 0).all()
    assert loss[1] == inf and torch.isfinite(dX[1]).all() and dX[1, 3] < 0
    assert torch.isfinite(loss[2]) and (dX[2, 40:] == 0).all()
    assert torch.isnan(loss[3]) and torch.isnan(dX[3]).all()
    assert torch.isfinite(loss[4]) and torch.isfinite(dX[4]).all()


def test_empty_tensors():
    for dtype in DTYPES:
        X = torch.empty(0, 47, dtype=dtype, device="cuda")
        e, t = torch.empty(0, device="cuda"), (torch.empty(0, 3, device="cuda"), torch.empty(0, 3, dtype=torch.int32, device="cuda"))
        sar.sar_logprob_fwd(X, torch.empty(0, dtype=torch.int32, device="cuda"), e, e, e, t)
        sar.sar_logprob_bwd(X, None, e, e, None, e, X)
        sar.sar_distill_fwd(X, t, 1.0, e, e)
        sar.sar_distill_bwd(X, t, 1.0, e, e, X)
