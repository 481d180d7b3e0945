"""Weight gradients by type over many rows: how far all of their entries together are off, against 64 bits.

A worst case's bound grows with the rows, and of 100 thousand of them a lost chunk is less.  Roundings are of either sign: the errors of sums of R
products x z go as sqrt(R).  In units of U sqrt(R) rms(x) rms(z), U = 2^-24 (a partial sum of r rows being of size sqrt(r) in units of a product):
  - fp32: products off by up to 2 U each                                                                                     up to 2
    a share of A chunks of 16 rows, a rounding of the sum so far a chunk, 0.3 U of a number of size sqrt(16 a), a = 1 .. A, together over
    R / (16 A) shares: 0.3 sqrt(A / 2), with A <= 256 (shares of 4096 rows at these sizes)                                    up to 4
    the shares' sums, up to 768 of them by eights: a hundred additions behind each other of numbers up to sqrt(R), 0.3 sqrt(100)    3
    what the matrix unit cuts of 16 products' sum, up to six units of size sqrt(16) a chunk, turned with every other chunk    up to 6
  together, as the errors are of either sign, below sqrt(4 + 16 + 9 + 36) = 8; held to 16.
  - bf16: products added in the matrix unit, a unit cut (2 U at most) for eight of them, its sign turned every 128 rows: a block of 16 cuts of a
    number of size sqrt(r) that no block of the other sign takes back, and what two neighbouring blocks differ by: 16 + sqrt(A) of a share; held to 32.
"""
import numpy as np
import pytest
import torch

from tests import nodewise as nw

F32, BF16 = torch.float32, torch.bfloat16
KINDS = [(F32, False), (F32, True), (BF16, False), (BF16, True)]       # rows' type; X in 8 bits
HELD = {F32: 16, BF16: 32}


def rms(v):
    return float(np.sqrt(np.mean(np.square(v))))


def sums_are_close(got, x, z, dtype):
    """Entries all together, and none of them far beyond the others (of 65536 normal ones the largest is below 5 deviations)."""
    held = HELD[dtype] * nw.U * np.sqrt(len(x)) * rms(x) * rms(z)
    off = got - x.T @ z
    return rms(off) <= held and np.abs(off).max() <= 6 * held


# ---- the bound itself, on the host

def chunk_sums(x, z, cut=False):
    """Sums in 32 bits, 16 rows at a time one after the other in shares of 1024 rows; cut: each towards minus infinity."""
    total = np.zeros((x.shape[1], z.shape[1]), np.float32)
    for lo in range(0, len(x), 1024):
        share = np.zeros_like(total)
        for r in range(lo, min(lo + 1024, len(x)), 16):
            s = share.astype(np.float64) + (x[r:min(r + 16, lo + 1024)].T @ z[r:min(r + 16, lo + 1024)])
            share = s.astype(np.float32)
            if cut:
                share = np.where(share.astype(np.float64) > s, np.nextafter(share, np.float32(-np.inf)), share)
        total += share
    return total.astype(np.float64)


def pieces(v, count):
    """v as the sum of so many bf16 values."""
    left, out = torch.from_numpy(v), 0.0
    for _ in range(count):
        p = left.to(BF16).double()
        out, left = out + p, left - p
    return out.numpy()


def mistakes(x, z):
    yield "one piece of bf16", chunk_sums(pieces(x, 1), pieces(z, 1))
    yield "one piece of the second operand", chunk_sums(x, pieces(z, 1))
    yield "two pieces of bf16", chunk_sums(pieces(x, 2), pieces(z, 2))
    for name, rows in (("a chunk", slice(4000, 4016)), ("a row", slice(4000, 4001)), ("the last row", slice(len(x) - 1, len(x)))):
        part = x.copy()
        part[rows] = 0
        yield name + " lost", chunk_sums(part, z)
        yield name + " twice", chunk_sums(x + (x - part), z)
    yield "sums cut to one side", chunk_sums(x, z, cut=True)
    tile = chunk_sums(x, z)
    tile[:32, :32] -= x[4000:4016, :32].T @ z[4000:4016, :32]
    yield "a chunk lost in one tile", tile


def test_what_the_bound_lets_through_and_what_it_does_not():
    rng = np.random.default_rng(4)
    x, z = (rng.standard_normal((170_000, 64)).astype(np.float32).astype(np.float64) for _ in range(2))
    assert sums_are_close(chunk_sums(x, z), x, z, F32) and sums_are_close(chunk_sums(pieces(x, 3), pieces(z, 3)), x, z, F32)
    assert [name for name, got in mistakes(x, z) if sums_are_close(got, x, z, F32)] == []
    x, z = pieces(x, 1), pieces(z, 1)                              # bf16 rows: nothing to lose but rows
    assert sums_are_close(chunk_sums(x, z), x, z, BF16)
    assert [name for name, got in mistakes(x, z) if "piece" not in name and sums_are_close(got, x, z, BF16)] == []


# ---- the kernels: every tile that takes weights, with types of one row, of 15 and of 33 among large ones

@pytest.mark.gpu
@pytest.mark.parametrize("dtype,packed", KINDS)
@pytest.mark.parametrize("n,K,F", [(270_001, 256, 256), (270_001, 201, 70), (270_001, 100, 250), (120_001, 100, 100), (60_001, 128, 47),
                                   (60_001, 40, 100), (9001, 256, 256), (3000, 300, 200), (1000, 256, 256)])
def test_entries_all_together(n, K, F, dtype, packed):
    from paper_2111_06483_amd import sar
    g = torch.Generator().manual_seed(n + K)
    X, dZ = torch.randn(n, K, generator=g).to(dtype).cuda(), torch.randn(n, F, generator=g).to(dtype).cuda()
    a = n // 3
    ends = [5, a, a, a + 1, a + 16, a + 49, n - 7]
    W, dW = torch.empty(6, K, F, device="cuda"), torch.empty(6, K, F, device="cuda")
    rows, x = X, nw.f64(X)
    if packed:
        rows = sar.packed_empty(n, K)
        sar.sar_pack(X, rows)
        x = nw.unpack(rows[0].cpu().numpy(), rows[1].cpu().numpy(), K)
    work = torch.empty(sar.sar_linear_typed_workspace_bytes(n, K, F, 6), dtype=torch.uint8, device="cuda")
    sar.sar_linear_typed_bwd(rows, dZ, W, torch.tensor(ends, dtype=torch.int32, device="cuda"), False, dW, None, work)
    z, got = nw.f64(dZ), nw.f64(dW)
    for t, lo, hi in nw.spans(ends, n):
        if lo == hi:
            assert (got[t] == 0).all()
        else:
            assert sums_are_close(got[t], x[lo:hi], z[lo:hi], dtype), (t, lo, hi, rms(got[t] - x[lo:hi].T @ z[lo:hi]) / nw.U / np.sqrt(hi - lo))


# ---- which kernels take weight gradients and backward passes of several types, on both sides of the lines

LINES = [
    # so many rows a type: 256
    (2048, 64, 64, 8, ["k_typed_dw_few"], ["k_typed_few_bwd"]), (2049, 64, 64, 8, ["k_typed_dw<", "k_typed_sum"], ["k_typed_dw<", "k_typed_few"]),
    # 16384 rows, of however many types
    (16_384, 64, 64, 100, ["k_typed_dw_few"], ["k_typed_few_bwd"]), (16_385, 64, 64, 100, ["k_typed_dw<", "k_typed_sum"], ["k_typed_dw<", "k_typed_few"]),
    # the columns read anew by every 32 x 32 weights
    (1024, 1024, 1024, 2, ["k_typed_dw_few"], ["k_typed_dw_few", "k_typed_few"]), (1025, 1024, 1024, 5, ["k_typed_dw<", "k_typed_sum"], ["k_typed_dw<", "k_typed_few"]),
    # as many wavefronts of both products as the chip holds
    (2000, 256, 256, 8, ["k_typed_dw_few"], ["k_typed_few_bwd"]), (8000, 256, 256, 46, ["k_typed_dw_few"], ["k_typed_dw_few", "k_typed_few"]),
    # dX by its own kernels of many rows (blocks of 32 x 32 results)
    (10_000, 256, 64, 60, ["k_typed_dw_few"], ["k_typed_dw_few", "k_typed_lay", "k_typed_rows"]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("n,K,F,T,dw,both", LINES)
def test_which_kernels_take_several_types(n, K, F, T, dw, both):
    from paper_2111_06483_amd import sar
    from tests import gpu_util as gu
    g = torch.Generator().manual_seed(n)
    X, dZ, W = torch.randn(n, K, generator=g).cuda(), torch.randn(n, F, generator=g).cuda(), torch.randn(T, K, F, generator=g).cuda()
    ends = [n * t // T for t in range(T + 1)]
    ptr = torch.tensor(ends, dtype=torch.int32, device="cuda")
    work = torch.empty(sar.sar_linear_typed_workspace_bytes(n, K, F, T), dtype=torch.uint8, device="cuda")
    dW, dX = torch.empty_like(W), torch.empty_like(X)
    names = ("k_typed_dw_few", "k_typed_few_bwd", "k_typed_few", "k_typed_dw<", "k_typed_sum", "k_typed_lay", "k_typed_rows")
    ran = lambda fn: {next(k for k in names if k in line) for line in gu.kernels_of(fn).split("\n") if "k_typed" in line}
    kernels = ran(lambda: sar.sar_linear_typed_bwd(X, dZ, W, ptr, False, dW, None, work))
    assert kernels == set(dw), kernels
    kernels = ran(lambda: sar.sar_linear_typed_bwd(X, dZ, W, ptr, False, dW, dX, work))
    assert kernels - {"k_typed_sum"} == set(both), kernels
    x, z, w, got = nw.f64(X), nw.f64(dZ), nw.f64(W), nw.f64(dW)
    for t, lo, hi in nw.spans(ends, n):
        assert sums_are_close(got[t], x[lo:hi], z[lo:hi], F32), t
        want, size = z[lo:hi] @ w[t].T, np.abs(z[lo:hi]) @ np.abs(w[t]).T
        assert (np.abs(nw.f64(dX[lo:hi]) - want) <= (32 + F / 32) * 2 * nw.U * size).all(), t
