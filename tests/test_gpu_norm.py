"""Layer norm, forward and backward, against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2111_06483_amd import sar
from tests import nodewise as nw

pytestmark = pytest.mark.gpu
EPS = 1e-5
DTYPES = [torch.float32, torch.bfloat16]
# every number of lanes and pieces a row can have, on both sides of each line, whole and ragged
WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 16, 31, 32, 33, 47, 64, 65, 100, 128, 129, 200, 255, 256, 257, 400, 512, 513, 777, 1000, 1024, 1025, 2047, 2048,
          2049, 4096, 4100, 8191, 8192]


def inputs(n, D, dtype, seed=0):
    g = torch.Generator().manual_seed(seed * 7919 + n * 31 + D)
    X = torch.randn(n, D, generator=g) * (0.5 + torch.rand(n, 1, generator=g)) + torch.randn(n, 1, generator=g)
    dY = torch.randn(n, D, generator=g)
    gamma, beta = 1 + 0.1 * torch.randn(D, generator=g), 0.1 * torch.randn(D, generator=g)
    return X.to(dtype).cuda(), dY.to(dtype).cuda(), gamma.cuda(), beta.cuda()


def terms(D):
    """Additions behind a row's mean: a lane's values one after the other, the lanes by halves; a few more operations."""
    return min(D, 32) + 16


def check_fwd(X, gamma, beta, Y, stats, eps=EPS):
    x, D = nw.f64(X), X.shape[1]
    g = nw.f64(gamma) if gamma is not None else np.ones(D)
    b = nw.f64(beta) if beta is not None else np.zeros(D)
    y, mean, r = nw.norm_fwd(x, g, b, eps)
    size = np.abs(x).mean(1, keepdims=True)                      # the scale of the terms of the mean
    off_mean = terms(D) * nw.U * size
    # the variance's terms carry the mean's error twice; 1 / sqrt halves a relative error, its own two roundings
    dev = np.abs(x - mean)
    off_r = r * ((terms(D) + 8) * nw.U + (dev.mean(1, keepdims=True) * 2 * (off_mean + nw.U * size)) * r * r)
    if stats is not None:
        s = nw.f64(stats)
        assert (np.abs(s[:, :1] - mean) <= off_mean).all()
        assert (np.abs(s[:, 1:] - r) <= off_r).all()
    off = (off_mean * r + dev * off_r + 4 * nw.U * dev * r) * np.abs(g) + 2 * nw.U * np.abs(b)
    got = nw.f64(Y)
    assert (np.abs(got - y) <= off + nw.half_step(X.dtype)(np.abs(y) + off)).all()


def check_bwd(dY, x, stats, gamma, dX, dgamma, dbeta, before=(0.0, 0.0)):
    """stats as they were handed over: their own errors are the forward pass's."""
    dy, D, n = nw.f64(dY), dY.shape[1], dY.shape[0]
    s, g = nw.f64(stats), nw.f64(gamma) if gamma is not None else np.ones(dY.shape[1])
    dx, dg, db = nw.norm_bwd(dy, x, s[:, :1], s[:, 1:], g)
    h = np.abs((x - s[:, :1]) * s[:, 1:]) + 2 * nw.U * (np.abs(x) + np.abs(s[:, :1])) * s[:, 1:]
    d = np.abs(dy * g)
    size = d + d.mean(1, keepdims=True) + h * (d * h).mean(1, keepdims=True)
    if dX is not None:
        off = s[:, 1:] * (terms(D) + 16) * nw.U * size
        assert (np.abs(nw.f64(dX) - dx) <= off + nw.half_step(dY.dtype)(np.abs(dx) + off)).all()
    # a thread's rows one after the other (2048 workgroups and more than one row each), then 4 wavefronts, 32 slices ...
    many = n / 256 + 128
    if dgamma is not None:
        assert (np.abs(nw.f64(dgamma) - before[0] - dg) <= many * nw.U * ((np.abs(dy) * h).sum(0) + np.abs(before[0]))).all()
    if dbeta is not None:
        assert (np.abs(nw.f64(dbeta) - before[1] - db) <= many * nw.U * (np.abs(dy).sum(0) + np.abs(before[1]))).all()


def work_for(n, D):
    return torch.empty(sar.sar_layernorm_workspace_bytes(n, D), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_rows_of_every_width(D, dtype):
    n = 37 if D > 600 else 301
    X, dY, gamma, beta = inputs(n, D, dtype)
    Y, stats = torch.empty_like(X), torch.empty(n, 2, device="cuda")
    xp, yp = sar.packed_empty(n, D), sar.packed_empty(n, D)
    sar.sar_layernorm_fwd(X, gamma, beta, EPS, Y, stats, xp, yp)
    check_fwd(X, gamma, beta, Y, stats)
    for p, full in ((xp, X), (yp, Y)):                           # as if packed by a call of their own
        q, e = sar.packed_empty(n, D)
        sar.sar_pack(full, (q, e))
        assert torch.equal(q, p[0]) and torch.equal(e, p[1])
    dX, dg, db = torch.empty_like(X), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    work = work_for(n, D)
    sar.sar_layernorm_bwd(dY, X, stats, gamma, False, dX, dg, db, work)
    check_bwd(dY, nw.f64(X), stats, gamma, dX, dg, db)
    sar.sar_layernorm_bwd(dY, xp, stats, gamma, False, dX, dg, db, work)
    check_bwd(dY, nw.unpack(xp[0].cpu().numpy(), xp[1].cpu().numpy(), D), stats, gamma, dX, dg, db)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 31, 33, 1000, 70_001])
@pytest.mark.parametrize("D", [5, 64, 256])
def test_every_number_of_rows(n, D, dtype):
    X, dY, gamma, beta = inputs(n, D, dtype)
    Y, stats = torch.empty_like(X), torch.empty(n, 2, device="cuda")
    sar.sar_layernorm_fwd(X, gamma, beta, EPS, Y, stats)
    check_fwd(X, gamma, beta, Y, stats)
    dX, dg, db = torch.empty_like(X), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    sar.sar_layernorm_bwd(dY, X, stats, gamma, False, dX, dg, db, work_for(n, D))
    check_bwd(dY, nw.f64(X), stats, gamma, dX, dg, db)


@pytest.mark.parametrize("dtype", DTYPES)
def test_what_may_be_left_out_or_shared(dtype):
    n, D = 513, 100
    X, dY, gamma, beta = inputs(n, D, dtype)
    Y, stats = torch.empty_like(X), torch.empty(n, 2, device="cuda")
    sar.sar_layernorm_fwd(X, None, None, EPS, Y, stats)
    check_fwd(X, None, None, Y, stats)
    sar.sar_layernorm_fwd(X, gamma, None, 0.0, Y)
    check_fwd(X, gamma, None, Y, None, 0.0)
    Z = X.clone()
    sar.sar_layernorm_fwd(Z, gamma, None, 0.0, Z)
    assert torch.equal(Z, Y)
    work = work_for(n, D)
    full = [torch.empty_like(X), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")]
    sar.sar_layernorm_bwd(dY, X, stats, None, False, *full, work)
    check_bwd(dY, nw.f64(X), stats, None, *full)
    for left_out in range(3):
        part = [None if k == left_out else torch.empty_like(t) for k, t in enumerate(full)]
        sar.sar_layernorm_bwd(dY, X, stats, None, False, *part, work)
        assert all(p is None or torch.equal(p, f) for p, f in zip(part, full))
    sar.sar_layernorm_bwd(dY, X, stats, None, False, full[0], None, None, None)         # no parameters: no scratch
    over = dY.clone()                                            # dX in the place of dY, and of X
    sar.sar_layernorm_bwd(over, X, stats, None, False, over, None, None, None)
    assert torch.equal(over, full[0])
    over = X.clone()
    sar.sar_layernorm_bwd(dY, over, stats, None, False, over, None, None, None)
    assert torch.equal(over, full[0])


def test_gradients_added_to_what_is_there():
    for n in (3, 5000, 0):
        X, dY, gamma, beta = inputs(n, 48, torch.float32)
        _, mean, r = nw.norm_fwd(nw.f64(X), 1, 0, EPS)
        stats = torch.from_numpy(np.concatenate([mean, r], 1)).float().cuda()
        first = torch.randn(2, 48, generator=torch.Generator().manual_seed(n)).cuda()
        dg, db = first.clone().unbind(0)
        sar.sar_layernorm_bwd(dY, X, stats, gamma, True, torch.empty_like(X), dg, db, work_for(n, 48))
        check_bwd(dY, nw.f64(X), stats, gamma, None, dg, db, (nw.f64(first[0]), nw.f64(first[1])))
        sar.sar_layernorm_bwd(dY, X, stats, gamma, False, None, dg, db, work_for(n, 48))
        check_bwd(dY, nw.f64(X), stats, gamma, None, dg, db)


def test_gradient_by_differences():
    """dX, dgamma and dbeta against differences of the 64-bit forward function along random directions."""
    n, D = 40, 24
    X, dY, gamma, beta = inputs(n, D, torch.float32)
    Y, stats = torch.empty_like(X), torch.empty(n, 2, device="cuda")
    sar.sar_layernorm_fwd(X, gamma, beta, EPS, Y, stats)
    dX, dg, db = torch.empty_like(X), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    sar.sar_layernorm_bwd(dY, X, stats, gamma, False, dX, dg, db, work_for(n, D))
    x, dy, g, b = nw.f64(X), nw.f64(dY), nw.f64(gamma), nw.f64(beta)
    loss = lambda x, g, b: (nw.norm_fwd(x, g, b, EPS)[0] * dy).sum()
    rng, h = np.random.default_rng(5), 1e-5
    for _ in range(4):
        vx, vg, vb = rng.standard_normal(x.shape), rng.standard_normal(D), rng.standard_normal(D)
        for got, d in ((nw.f64(dX), (vx, 0, 0)), (nw.f64(dg), (0, vg, 0)), (nw.f64(db), (0, 0, vb))):
            v = [t for t in d if not np.isscalar(t)][0]
            slope = (loss(x + h * d[0], g + h * d[1], b + h * d[2]) - loss(x - h * d[0], g - h * d[1], b - h * d[2])) / (2 * h)
            # differences: h^2 times a third derivative; the kernel: some hundred roundings of terms of the sum's size
            assert abs((got * v).sum() - slope) <= 1e-7 * n * D + 128 * nw.U * np.abs(got * v).sum() * 8


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_that_are_constant_huge_or_not_finite(dtype):
    n, D = 9, 70
    X = torch.randn(n, D, generator=torch.Generator().manual_seed(3))
    X[0] = 0.0
    X[1] = 3.0
    X[2] *= 1e18
    X[3] *= 1e-18
    X[4, 7] = float("inf")
    X[5, 8] = float("nan")
    X = X.to(dtype).cuda()
    Y, stats = torch.empty_like(X), torch.empty(n, 2, device="cuda")
    sar.sar_layernorm_fwd(X, None, None, EPS, Y, stats)
    fine = [0, 1, 2, 3, 6, 7, 8]
    check_fwd(X[fine], None, None, Y[fine], stats[fine])
    assert not torch.isfinite(Y[4]).any() and not torch.isfinite(Y[5]).any()
    assert torch.isnan(Y[4]).all() and torch.isnan(Y[5]).all()
    # the rows beside them keep their gradients
    dY = torch.randn(n, D, generator=torch.Generator().manual_seed(4)).to(dtype).cuda()
    dX = torch.empty_like(X)
    sar.sar_layernorm_bwd(dY, X, stats, None, False, dX, None, None, None)
    check_bwd(dY[fine], nw.f64(X[fine]), stats[fine], None, dX[fine], None, None)
    assert torch.isnan(dX[4]).all() and torch.isnan(dX[5]).all()


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,D", [(2, 47), (100, 2100), (1024, 70), (1025, 70), (1000, 8192)])
def test_both_sides_of_few_rows(n, D, dtype, packed):
    """One launch for few rows, two for more; parameters alone, and dX in the place of an operand that the parameters need."""
    X, dY, gamma, beta = inputs(n, D, dtype)
    Y, stats = torch.empty_like(X), torch.empty(n, 2, device="cuda")
    p = sar.packed_empty(n, D, "cuda")
    sar.sar_layernorm_fwd(X, gamma, beta, EPS, Y, stats, p)
    if packed:
        sar.sar_unpack(p, X)
    x, work = nw.f64(X), work_for(n, D)
    dX, dg, db = torch.empty_like(X), torch.ones(D, device="cuda"), torch.ones(D, device="cuda")
    sar.sar_layernorm_bwd(dY, p if packed else X, stats, gamma, True, dX, dg, db, work)
    check_bwd(dY, x, stats, gamma, dX, dg, db, (1.0, 1.0))
    only = torch.empty(D, device="cuda")
    sar.sar_layernorm_bwd(dY, p if packed else X, stats, gamma, False, None, only, None, work)
    check_bwd(dY, x, stats, gamma, None, only, None)
    over = dY.clone()
    sar.sar_layernorm_bwd(over, p if packed else X, stats, gamma, False, over, dg, db, work)
    check_bwd(dY, x, stats, gamma, over, dg, db)
    if not packed:
        sar.sar_layernorm_bwd(dY, X, stats, gamma, False, X, dg, db, work)
        check_bwd(dY, x, stats, gamma, X, dg, db)


def test_the_same_in_every_run():
    X, dY, gamma, beta = inputs(100_003, 47, torch.float32)
    stats, Y = torch.empty(100_003, 2, device="cuda"), torch.empty_like(X)
    sar.sar_layernorm_fwd(X, gamma, beta, EPS, Y, stats)
    got = []
    for _ in range(3):
        dg, db = torch.empty(47, device="cuda"), torch.empty(47, device="cuda")
        sar.sar_layernorm_bwd(dY, X, stats, gamma, False, None, dg, db, work_for(100_003, 47))
        got.append((dg, db))
    assert all(torch.equal(a, b) for g in got[1:] for a, b in zip(g, got[0]))


def test_rows_that_begin_anywhere_and_neighbours():
    """Tensors at odd addresses; the values before and behind the outputs stay."""
    for dtype in DTYPES:
        n, D = 21, 39
        X, dY, gamma, beta = inputs(n, D, dtype)
        room = [torch.full((n * D + 7,), 5.0, dtype=dtype, device="cuda") for _ in range(4)]
        x, dy, y, dx = (r[3:3 + n * D].view(n, D) for r in room)
        x.copy_(X), dy.copy_(dY)
        stats = torch.empty(n, 2, device="cuda")
        params = torch.zeros(2 * D + 1, device="cuda")
        gm, bt = params[1:D + 1], params[D + 1:]
        gm.copy_(gamma), bt.copy_(beta)
        sar.sar_layernorm_fwd(x, gm, bt, EPS, y, stats)
        check_fwd(X, gamma, beta, y, stats)
        grads = torch.full((2 * D + 3,), 9.0, device="cuda")
        sar.sar_layernorm_bwd(dy, x, stats, gm, False, dx, grads[1:D + 1], grads[D + 2:2 * D + 2], work_for(n, D))
        check_bwd(dY, nw.f64(X), stats, gamma, dx, grads[1:D + 1], grads[D + 2:2 * D + 2])
        assert all(bool((r[:3] == 5).all()) and bool((r[-4:] == 5).all()) for r in room)
        assert float(grads[0]) == 9 and float(grads[D + 1]) == 9 and float(grads[-1]) == 9
