"""Transforms with a weight per node type, and weight gradients from rows in 8 bits, against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2111_06483_amd import sar
from tests import nodewise as nw

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DTYPES = [F32, BF16]
KINDS = [(F32, False), (F32, True), (BF16, False), (BF16, True)]       # rows' type; X in 8 bits


def inputs(n, K, F, T, dtype, seed=0):
    g = torch.Generator().manual_seed(seed * 104729 + n * 131 + K * 17 + F)
    X = torch.randn(n, K, generator=g).to(dtype).cuda()
    dZ = torch.randn(n, F, generator=g).to(dtype).cuda()
    W = (torch.randn(T, K, F, generator=g) / K ** 0.5).cuda()
    return X, dZ, W


def ptr_of(ends):
    return torch.tensor(ends, dtype=torch.int32, device="cuda")


def work_for(n, K, F, T):
    return torch.empty(sar.sar_linear_typed_workspace_bytes(n, K, F, T), dtype=torch.uint8, device="cuda")


def packed_of(X):
    p = sar.packed_empty(*X.shape)
    sar.sar_pack(X, p)
    return p, nw.unpack(p[0].cpu().numpy(), p[1].cpu().numpy(), X.shape[1])


def rows_off(size, C, dtype):
    """How far a product of C terms may be off, `size` = sum |a||b|: fp32 sums of 32 exact products cut at up to 24 places (a unit
    each) and added, the weights' 16 bits and a unit for each of the C/8 additions where rows are bf16; the rounding of the result."""
    if dtype == F32:
        return (32 + C / 32) * 2 * nw.U * size
    return (2.0 ** -16 + C / 8 * 2 * nw.U) * size


def dw_off(size, rows):
    """Sums of up to 64 products from zero, cut; a workgroup's sums one after the other, then the workgroups'."""
    return (64 + rows / 32) * 2 * nw.U * size


def check_rows(A, W, Z, spans, dtype, trans):
    """Z = A W_t (trans: A W_t^T) on the types' rows."""
    a, w, z = nw.f64(A), nw.f64(W), nw.f64(Z)
    for t, lo, hi in spans:
        m = w[t].T if trans else w[t]
        want, size = a[lo:hi] @ m, np.abs(a[lo:hi]) @ np.abs(m)
        off = rows_off(size, m.shape[0], dtype)
        tol = off + (nw.half_step(dtype)(np.abs(want) + off) if dtype == BF16 else 0)
        assert (np.abs(z[lo:hi] - want) <= tol).all(), (t, lo, hi)


def check_dw(x, dZ, dW, spans, before=None):
    d, got = nw.f64(dZ), nw.f64(dW)
    for t, lo, hi in spans:
        want, size = x[lo:hi].T @ d[lo:hi], np.abs(x[lo:hi]).T @ np.abs(d[lo:hi])
        if before is not None:
            want, size = want + before[t], size + np.abs(before[t])
        assert (np.abs(got[t] - want) <= dw_off(size, hi - lo)).all(), (t, lo, hi)


def check_all(n, K, F, ends, dtype, packed, accumulate=False):
    T = len(ends) - 1
    X, dZ, W = inputs(n, K, F, T, dtype)
    ptr, work, spans = ptr_of(ends), work_for(n, K, F, T), nw.spans(ends, n)
    outside = np.ones(n, bool)
    for _, lo, hi in spans:
        outside[lo:hi] = False
    Z = torch.full((n, F), 3.0, dtype=dtype, device="cuda")
    sar.sar_linear_typed_fwd(X, W, ptr, Z, work)
    check_rows(X, W, Z, spans, dtype, False)
    dX = torch.full((n, K), 3.0, dtype=dtype, device="cuda")
    p, x = packed_of(X) if packed else (X, nw.f64(X))
    first = torch.randn(T, K, F, generator=torch.Generator().manual_seed(9)).cuda()
    dW = first.clone()
    sar.sar_linear_typed_bwd(p, dZ, W, ptr, accumulate, dW, dX, work)
    check_rows(dZ, W, dX, spans, dtype, True)
    check_dw(x, dZ, dW, spans, nw.f64(first) if accumulate else None)
    assert (nw.f64(Z)[outside] == 3).all() and (nw.f64(dX)[outside] == 3).all()
    return Z, dW, dX


# widths at which tiles, pieces and chunks end, whole and ragged
SHAPES = [(1, 1), (1, 40), (3, 2), (4, 4), (7, 9), (8, 8), (16, 47), (31, 33), (32, 64), (47, 65), (63, 100), (64, 129), (100, 256), (128, 128), (129, 31),
          (200, 47), (255, 257), (256, 256), (300, 200), (400, 130), (513, 20), (520, 520)]


@pytest.mark.parametrize("dtype,packed", KINDS)
@pytest.mark.parametrize("K,F", SHAPES)
def test_shapes(K, F, dtype, packed):
    check_all(331, K, F, [0, 100, 101, 101, 330], dtype, packed)


@pytest.mark.parametrize("dtype,packed", KINDS)
@pytest.mark.parametrize("n,K,F", [(140_003, 256, 256), (270_001, 100, 250), (270_001, 201, 70)])
def test_weight_gradients_by_the_widest_tiles(n, K, F, dtype, packed):
    X, dZ, W = inputs(n, K, F, 3, dtype)
    p, x = packed_of(X) if packed else (X, nw.f64(X))
    ends = [5, 100_000, 100_000, n - 7]
    dW = torch.empty_like(W)
    sar.sar_linear_typed_bwd(p, dZ, W, ptr_of(ends), False, dW, None, work_for(n, K, F, 3))
    check_dw(x, dZ, dW, nw.spans(ends, n))


@pytest.mark.parametrize("dtype,packed", KINDS)
@pytest.mark.parametrize("K,F", [(1, 1), (1, 40), (3, 2), (7, 9), (16, 47), (31, 33), (47, 65), (63, 100), (64, 129), (129, 31)])
def test_shapes_by_the_kernels_of_many_rows(K, F, dtype, packed):
    """Ragged widths where the calls of few rows are not taken: both products of rows, and the weights' gradients in shares."""
    check_all(85_003, K, F, [0, 100, 101, 101, 40_000, 85_000], dtype, packed)


@pytest.mark.parametrize("dtype,packed", KINDS)
@pytest.mark.parametrize("K,F", [(100, 256), (256, 256), (72, 60), (4, 264), (520, 100), (8, 1000), (300, 130), (99, 256), (250, 88)])
def test_many_rows(K, F, dtype, packed):
    """Enough rows for the wide tiles, several chunks a workgroup, types that end anywhere in a workgroup's rows."""
    n = 140_003
    check_all(n, K, F, [0, 5, 5, 40_000, 40_001, 90_017, n - 7], dtype, packed)


@pytest.mark.parametrize("dtype,packed", KINDS)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 255, 256, 257, 1000])
def test_every_number_of_rows(n, dtype, packed):
    check_all(n, 40, 24, [0, n], dtype, packed)
    check_all(n, 40, 24, [0, n // 3, n // 3, n], dtype, packed, accumulate=True)


@pytest.mark.parametrize("dtype,packed", KINDS)
def test_types_without_rows_and_rows_without_a_type(dtype, packed):
    check_all(90, 33, 20, [0, 0, 0, 0], dtype, packed)
    check_all(90, 33, 20, [0, 0, 50, 50, 50, 80], dtype, packed)
    check_all(90, 33, 20, [10, 30, 80], dtype, packed, accumulate=True)
    check_all(90, 33, 20, [90, 90], dtype, packed)


@pytest.mark.parametrize("dtype", DTYPES)
def test_more_types_than_a_wavefront_has_lanes(dtype):
    rng = np.random.default_rng(1)
    sizes = rng.integers(0, 40, 150)
    sizes[60:70] = 0
    ends = np.concatenate([[0], np.cumsum(sizes)])
    check_all(int(ends[-1]) + 3, 24, 40, ends.tolist(), dtype, False)
    check_all(int(ends[-1]), 24, 40, ends.tolist(), dtype, True)


def test_bounds_that_leave_the_rows_are_cut():
    check_all(50, 20, 20, [-5, 10, 70, 2_000_000_000], F32, False)


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_rows(dtype):
    X, dZ, W = inputs(0, 12, 20, 2, dtype)
    ptr, work = ptr_of([0, 0, 0]), work_for(0, 12, 20, 2)
    sar.sar_linear_typed_fwd(X, W, ptr, torch.empty(0, 20, dtype=dtype, device="cuda"), work)
    dW = torch.ones_like(W)
    sar.sar_linear_typed_bwd(X, dZ, W, ptr, True, dW, torch.empty_like(X), work)
    assert bool((dW == 1).all())
    sar.sar_linear_typed_bwd(X, dZ, W, ptr, False, dW, torch.empty_like(X), work)
    assert bool((dW == 0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,K,F", [(1, 5, 7), (700, 100, 256), (50_001, 47, 130)])
def test_plain_transform_from_packed_rows(n, K, F, dtype):
    X, dZ, W = inputs(n, K, F, 1, dtype)
    p, x = packed_of(X)
    work = work_for(n, K, F, 1)
    dW, dX = torch.empty(K, F, device="cuda"), torch.empty_like(X)
    sar.sar_linear_bwd_packed(p, dZ, W[0], False, dW, dX, work)
    check_dw(x, dZ, dW[None], [(0, 0, n)])
    check_rows(dZ, W, dX, [(0, 0, n)], dtype, True)
    once = dW.clone()
    sar.sar_linear_bwd_packed(p, dZ, W[0], True, dW, None, work)         # added: the same sums once more
    assert torch.equal(dW, once + once)
    only = torch.empty_like(dX)
    sar.sar_linear_bwd_packed(None, dZ, W[0], False, None, only, work)
    assert torch.equal(only, dX)


def test_packed_rows_are_bf16_rows():
    """A packed row's values are bf16 values: dW from them is that from bf16 rows, bit for bit."""
    X, dZ, W = inputs(3001, 90, 70, 1, BF16)
    p, _ = packed_of(X)
    same = torch.empty_like(X)
    sar.sar_unpack(p, same)
    ptr, work = ptr_of([0, 3001]), work_for(3001, 90, 70, 1)
    a, b = torch.empty_like(W), torch.empty_like(W)
    sar.sar_linear_typed_bwd(p, dZ, W, ptr, False, a, None, work)
    sar.sar_linear_typed_bwd(same, dZ, W, ptr, False, b, None, work)
    assert torch.equal(a, b)


def test_sums_lean_to_no_side():
    """Sums of 400 thousand products of one sign's mean error: cut sums would all be too small."""
    n, K, F = 400_000, 40, 40
    for dtype, packed in KINDS:
        X, dZ, W = inputs(n, K, F, 1, dtype)
        p, x = packed_of(X) if packed else (X, nw.f64(X))
        dW = torch.empty_like(W)
        sar.sar_linear_typed_bwd(p, dZ, W, ptr_of([0, n]), False, dW, None, work_for(n, K, F, 1))
        d = nw.f64(dZ)
        off = nw.f64(dW)[0] - x.T @ d
        # 1600 sums of n terms: their errors' mean is zero within 4 of its deviations, and each is some roundings of the sum's size
        assert abs(off.mean()) <= 4 * off.std() / 40 + 1e-12
        assert off.std() <= 1e-6 * np.sqrt(n)


def with_specials(a, b):
    """a b where both have infinities and NaN: the finite part by a product, every special number's terms one by one."""
    fa, fb = np.where(np.isfinite(a), a, 0.0), np.where(np.isfinite(b), b, 0.0)
    want, size = fa @ fb, np.abs(fa) @ np.abs(fb)
    with np.errstate(invalid="ignore"):
        for i, k in np.argwhere(~np.isfinite(a)):
            want[i] += a[i, k] * b[k]
        for k, j in np.argwhere(~np.isfinite(b)):
            rest = np.isfinite(a[:, k])
            want[rest, j] += a[rest, k] * b[k, j]
    return want, size


# (rows, widths): calls of few rows, and of many
@pytest.mark.parametrize("n,K,F", [(300, 40, 50), (2000, 256, 130), (70_000, 101, 256), (70_000, 256, 128)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_infinities_and_nan_stay_where_they_belong(n, K, F, dtype):
    X, dZ, W = inputs(n, K, F, 2, dtype)
    X[7, 3] = float("inf")
    X[n - 100, 5] = float("nan")
    dZ[9, 4] = -float("inf")
    dZ[n // 2, 0] = float("inf")
    W = W.clone()
    W[1, 6, 8] = float("inf")
    ends = [0, n // 2, n]
    ptr, work = ptr_of(ends), work_for(n, K, F, 2)
    Z, dX, dW = torch.empty(n, F, dtype=dtype, device="cuda"), torch.empty_like(X), torch.empty_like(W)
    sar.sar_linear_typed_fwd(X, W, ptr, Z, work)
    sar.sar_linear_typed_bwd(X, dZ, W, ptr, False, dW, dX, work)
    x, d, w = nw.f64(X), nw.f64(dZ), nw.f64(W)
    for t, lo, hi in nw.spans(ends, n):
        for got, a, b, rounded in ((nw.f64(Z)[lo:hi], x[lo:hi], w[t], True), (nw.f64(dX)[lo:hi], d[lo:hi], w[t].T, True),
                                   (nw.f64(dW)[t], x[lo:hi].T, d[lo:hi], False)):
            want, size = with_specials(a, b)
            fine = np.isfinite(want)
            assert np.array_equal(got[~fine], want[~fine], equal_nan=True)
            off = rows_off(size, a.shape[1], dtype) if rounded else dw_off(size, a.shape[1])
            # (a tile that is taken again adds its products one by one)
            off = off + a.shape[1] * nw.U * size
            if rounded and dtype == BF16:
                off = off + nw.half_step(dtype)(np.abs(np.where(fine, want, 0)) + off)
            assert (np.abs(got - want)[fine] <= off[fine]).all()


def test_the_largest_and_the_smallest_numbers():
    """fp32 values whose pieces round up to infinity, and values near 2^-110."""
    n, K, F = 70, 40, 36
    X, dZ, W = inputs(n, K, F, 1, F32)
    X, dZ = torch.zeros_like(X), torch.zeros_like(dZ)
    X[3, 2] = torch.finfo(F32).max
    X[4, 5] = 2.0 ** -100 * 1.7
    dZ[3, 1] = 0.25
    dZ[4, 6] = 1.3
    W = torch.zeros_like(W)
    W[0, 2, 3] = 0.5
    W[0, 5, 7] = 1.9
    ptr, work = ptr_of([0, n]), work_for(n, K, F, 1)
    Z, dW = torch.empty(n, F, device="cuda"), torch.empty_like(W)
    sar.sar_linear_typed_fwd(X, W, ptr, Z, work)
    sar.sar_linear_typed_bwd(X, dZ, W, ptr, False, dW, None, work)
    for got, want in ((nw.f64(Z), nw.f64(X) @ nw.f64(W)[0]), (nw.f64(dW)[0], nw.f64(X).T @ nw.f64(dZ))):
        assert (np.abs(got - want) <= 2 * nw.U * 2 * np.abs(want)).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_tensors_that_begin_anywhere_and_neighbours(dtype):
    n, K, F, ends = 77, 37, 29, [0, 30, 70]
    X, dZ, W = inputs(n, K, F, 2, dtype)
    odd = lambda t, dt: torch.full((t.numel() + 5,), 6.0, dtype=dt, device="cuda")
    place = lambda buf, t: buf[1:1 + t.numel()].view(t.shape)
    room = {k: odd(t, t.dtype) for k, t in (("x", X), ("dz", dZ), ("w", W), ("dx", X), ("z", dZ), ("dw", W))}
    v = {k: place(room[k], t) for k, t in (("x", X), ("dz", dZ), ("w", W), ("dx", X), ("z", dZ), ("dw", W))}
    v["x"].copy_(X), v["dz"].copy_(dZ), v["w"].copy_(W)
    ptr, work, spans = ptr_of(ends), work_for(n, K, F, 2), nw.spans(ends, n)
    sar.sar_linear_typed_fwd(v["x"], v["w"], ptr, v["z"], work)
    sar.sar_linear_typed_bwd(v["x"], v["dz"], v["w"], ptr, False, v["dw"], v["dx"], work)
    check_rows(X, W, v["z"], spans, dtype, False)
    check_rows(dZ, W, v["dx"], spans, dtype, True)
    check_dw(nw.f64(X), dZ, v["dw"], spans)
    assert all(float(r[0]) == 6 and bool((r[-4:] == 6).all()) for r in room.values())


# Which kernels take a call, on both sides of the lines.
@pytest.mark.parametrize("n,K,F,dtype,fwd,dw", [
    (1000, 128, 128, BF16, "k_typed_few", "k_typed_dw_few"), (1024, 64, 64, F32, "k_typed_few", "k_typed_dw_few"),
    (1025, 64, 64, F32, "k_typed_few", "k_typed_dw<"), (1500, 512, 512, F32, "k_typed_few", "k_typed_dw<"), (40_000, 64, 64, F32, "k_typed_few", "k_typed_dw<"),
    (41_000, 64, 64, F32, "k_typed_rows<float, 2,", "k_typed_dw<"), (24_500, 100, 256, F32, "k_typed_rows<float, 2,", "k_typed_dw<"),
    (24_600, 100, 256, BF16, "k_typed_rows<sar::bf16_t, 4,", "k_typed_dw<"), (33_000, 102, 256, F32, "k_typed_rows<float, 8,", "k_typed_dw<"),
    (70_000, 104, 256, BF16, "k_typed_rows<sar::bf16_t, 8,", "k_typed_dw<"), (66_000, 256, 100, F32, "k_typed_rows<float, 4,", "k_typed_dw<")])
def test_which_kernels_run(n, K, F, dtype, fwd, dw):
    from tests import gpu_util as gu
    X, dZ, W = inputs(n, K, F, 1, dtype)
    ptr, work, Z, dW = ptr_of([0, n]), work_for(n, K, F, 1), torch.empty(n, F, dtype=dtype, device="cuda"), torch.empty_like(W)
    names = gu.kernels_of(lambda: sar.sar_linear_typed_fwd(X, W, ptr, Z, work))
    assert fwd in names and ("k_typed_few" in names) != ("k_typed_rows" in names), names
    names = gu.kernels_of(lambda: sar.sar_linear_typed_bwd(X, dZ, W, ptr, False, dW, None, work))
    assert dw in names, names
    check_rows(X, W, Z, [(0, 0, n)], dtype, False)
    check_dw(nw.f64(X), dZ, dW, [(0, 0, n)])


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_rows_that_begin_anywhere(dtype):
    """The first value off a 16-byte boundary."""
    n, K, F = 70_000, 128, 256
    X, dZ, W = inputs(n, K, F, 1, dtype)
    room = torch.empty(n * K + 1, dtype=dtype, device="cuda")
    x = room[1:].view(n, K)
    x.copy_(X)
    ptr, work, Z = ptr_of([0, n]), work_for(n, K, F, 1), torch.empty(n, F, dtype=dtype, device="cuda")
    sar.sar_linear_typed_fwd(x, W, ptr, Z, work)
    check_rows(X, W, Z, [(0, 0, n)], dtype, False)


@pytest.mark.parametrize("n,K,F,ends", [(1, 40, 30, [0, 1]), (90, 200, 140, [0, 30, 30, 80]), (600, 100, 300, [0, 600]), (2000, 400, 64, [0, 900, 2000]),
                                        (900, 256, 256, [0, 20, 900]), (5000, 64, 64, [0, 2500, 5000])])
@pytest.mark.parametrize("dtype,packed", KINDS)
def test_one_call_for_both_products_and_one_for_each(n, K, F, ends, dtype, packed):
    """The same bits, whichever launch they come from; also with dX in the place of X, which dW still has to read."""
    T = len(ends) - 1
    X, dZ, W = inputs(n, K, F, T, dtype)
    ptr, work, p = ptr_of(ends), work_for(n, K, F, T), packed_of(X)[0] if packed else X
    dW, dX = torch.empty_like(W), torch.zeros_like(X)
    sar.sar_linear_typed_bwd(p, dZ, W, ptr, False, dW, dX, work)
    dW1, dX1 = torch.empty_like(W), torch.zeros_like(X)
    sar.sar_linear_typed_bwd(p, dZ, W, ptr, False, dW1, None, work)
    sar.sar_linear_typed_bwd(None, dZ, W, ptr, False, None, dX1, work)
    assert torch.equal(dW, dW1) and torch.equal(dX, dX1)
    if not packed:
        X[ends[-1]:] = 0
        sar.sar_linear_typed_bwd(X, dZ, W, ptr, False, dW1, X, work)
        assert torch.equal(dW, dW1) and torch.equal(dX, X)
    if packed and T == 1:
        dW2, dX2 = torch.empty_like(W[0]), torch.empty_like(X)
        sar.sar_linear_bwd_packed(p, dZ, W[0], False, dW2, dX2, work)
        assert torch.equal(dW2, dW[0])


def test_the_same_in_every_run():
    n = 20_011
    got = [check_all(n, 100, 64, [0, 7000, 7001, n], F32, True) for _ in range(2)]
    assert all(torch.equal(a, b) for a, b in zip(*got))
