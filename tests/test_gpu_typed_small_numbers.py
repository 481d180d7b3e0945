"""Products by type of the smallest and of the largest numbers, against 64 bits: an operand keeps its bits whatever its size."""
import numpy as np
import pytest
import torch

from paper_2111_06483_amd import sar
from tests import nodewise as nw

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
# calls of few rows, and of many: every kernel of rows, and of weight gradients
SIZES = [(1, 40, 50), (300, 40, 50), (2000, 256, 130), (42_000, 60, 64), (70_000, 101, 256), (140_000, 256, 128)]
# sizes of one operand and the other: around the smallest whose last bit is a bf16 value, the smallest normal number (randn goes below it), numbers
# of few bits; and sizes and sums that are large, up to the largest numbers
SIZES_OF = [(-111, 60), (-122, 60), (-126, 60), (-140, 60), (102, -60), (110, -60), (124, -100), (60, 20)]


def numbers(n, K, F, dtype, seed):
    g = torch.Generator().manual_seed(seed * 7 + n + K + F)
    rn = lambda *s: torch.randn(*s, generator=g)
    return rn(n, K), rn(n, F), rn(2, K, F) / K ** 0.5


def scaled(t, power, dtype):
    """t 2^power (32 bits hold 2^power down to 2^-149), rounded to dtype."""
    return (t.double() * 2.0 ** power).to(F32).to(dtype).cuda()


def close(got, a, b, dtype, terms):
    """Sums of `terms` products, each formed within 2^-23 and added with a rounding or a cut of the sum so far (one by one in a result that is
    formed again); numbers below the normal ones are rounded to 2^-149, or to bf16's 2^-133."""
    want, size = a @ b, np.abs(a) @ np.abs(b)
    off = (32 + terms / 32) * 2 * nw.U * size
    if max(np.abs(v).max(initial=0) for v in (a, b)) > 2.0 ** 100 or size.max(initial=0) > 2.0 ** 78:
        off = off + min(terms, 2048) * nw.U * size             # (a workgroup has no more rows than that here)
    if dtype == BF16:
        # a weight of two bf16 pieces: 16 bits, or, where the second piece is below bf16's smallest value 2^-133, within half of that
        off = off + 2.0 ** -16 * size + 2.0 ** -134 * np.abs(a).sum(1, keepdims=True) + terms / 8 * 2 * nw.U * size
        off = off + nw.HALF[BF16] * (np.abs(want) + off) + 2.0 ** -134
    assert (np.abs(nw.f64(got) - want) <= off + 2.0 ** -149).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("power,other", SIZES_OF)
@pytest.mark.parametrize("n,K,F", SIZES)
def test_rows_times_weights(n, K, F, power, other, dtype):
    """Small rows times large weights, and the other way round; forward and back."""
    X, dZ, W = numbers(n, K, F, dtype, 1)
    ends = [0, n // 3, n]
    ptr = torch.tensor(ends, dtype=torch.int32, device="cuda")
    work = torch.empty(sar.sar_linear_typed_workspace_bytes(n, K, F, 2), dtype=torch.uint8, device="cuda")
    for rows_power, w_power in ((power, other), (other, power)):
        x, d, w = scaled(X, rows_power, dtype), scaled(dZ, rows_power, dtype), scaled(W, w_power, F32)
        Z, dX = torch.empty(n, F, dtype=dtype, device="cuda"), torch.empty(n, K, dtype=dtype, device="cuda")
        sar.sar_linear_typed_fwd(x, w, ptr, Z, work)
        sar.sar_linear_typed_bwd(None, d, w, ptr, False, None, dX, work)
        for t, lo, hi in nw.spans(ends, n):
            close(Z[lo:hi], nw.f64(x[lo:hi]), nw.f64(w[t]), dtype, K)
            close(dX[lo:hi], nw.f64(d[lo:hi]), nw.f64(w[t]).T, dtype, F)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("power,other", SIZES_OF)
@pytest.mark.parametrize("n,K,F", SIZES)
def test_weight_gradients(n, K, F, power, other, dtype, packed):
    X, dZ, W = numbers(n, K, F, dtype, 2)
    ends = [0, n // 3, n]
    ptr = torch.tensor(ends, dtype=torch.int32, device="cuda")
    work = torch.empty(sar.sar_linear_typed_workspace_bytes(n, K, F, 2), dtype=torch.uint8, device="cuda")
    for x_power, z_power in ((power, other), (other, power)):
        x, d = scaled(X, x_power, dtype), scaled(dZ, z_power, dtype)
        rows, values = x, nw.f64(x)
        if packed:
            rows = sar.packed_empty(n, K)
            sar.sar_pack(x, rows)
            values = nw.unpack(rows[0].cpu().numpy(), rows[1].cpu().numpy(), K)
        dW = torch.empty(2, K, F, device="cuda")
        sar.sar_linear_typed_bwd(rows, d, W.cuda(), ptr, False, dW, None, work)
        for t, lo, hi in nw.spans(ends, n):
            close(dW[t], values[lo:hi].T, nw.f64(d[lo:hi]), F32, hi - lo)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("power,other", SIZES_OF)
@pytest.mark.parametrize("n,K,F", [(1, 40, 50), (300, 100, 256), (1000, 256, 256), (30_000, 100, 256)])
def test_errors_from_packed_rows_are_those_of_the_transform(n, K, F, power, other, dtype):
    """dX of sar_linear_bwd_packed beside that of sar_linear_bwd, on both sides of few rows."""
    X, dZ, W = numbers(n, K, F, dtype, 3)
    d, w = scaled(dZ, power, dtype), scaled(W[0], other, F32)
    p = sar.packed_empty(n, K)
    sar.sar_pack(X.to(dtype).cuda(), p)
    dW, dX, plain = torch.empty(K, F, device="cuda"), torch.empty(n, K, dtype=dtype, device="cuda"), torch.empty(n, K, dtype=dtype, device="cuda")
    work = torch.empty(sar.sar_linear_typed_workspace_bytes(n, K, F, 1), dtype=torch.uint8, device="cuda")
    sar.sar_linear_bwd_packed(p, d, w, False, dW, dX, work)
    sar.sar_linear_bwd(None, d, w, None, plain, torch.empty(sar.sar_linear_workspace_bytes(n, K, F), dtype=torch.uint8, device="cuda"))
    for got in (dX, plain):
        close(got, nw.f64(d), nw.f64(w).T, dtype, F)
