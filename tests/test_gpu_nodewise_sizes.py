"""The node-wise operators at the ends of their documented sizes: tensors of more than 2^31 values, the widest weights, the most types."""
import numpy as np
import pytest
import torch

from paper_2111_06483_amd import sar
from tests import nodewise as nw

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5


def work_for(n, K, F, T):
    return torch.empty(sar.sar_linear_typed_workspace_bytes(n, K, F, T), dtype=torch.uint8, device="cuda")


def rows_off(size, C, dtype):
    """As many cuts and roundings of the sum so far as it has products by eights, products to within 2^-23; the weights' 16 bits where rows are bf16."""
    return (32 + C / 32) * 2 * nw.U * size if dtype == F32 else (2.0 ** -16 + C / 8 * 2 * nw.U) * size


def rows_close(got, a, b, dtype):
    want, size = a @ b, np.abs(a) @ np.abs(b)
    off = rows_off(size, a.shape[1], dtype)
    if dtype == BF16:
        off = off + nw.half_step(dtype)(np.abs(want) + off)
    assert (np.abs(nw.f64(got) - want) <= off).all()


def test_offsets_beyond_32_bits():
    """Layer norm, both packed forms, products by type and their backward passes on 2.15 thousand million values; rows at the ends and around 2^31 values
    and 2^32 bytes, and the sums over all rows."""
    n, K, F = 4_200_001, 512, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    rn = lambda *s, dtype=BF16: torch.randn(*s, dtype=dtype, device="cuda", generator=g)
    X, gamma, beta = rn(n, K), 1 + 0.1 * rn(K, dtype=F32), 0.1 * rn(K, dtype=F32)
    assert n * K > 1 << 31
    at = torch.tensor(sorted({r + d for r in (1, (1 << 31) // K, (1 << 30) // K, n - 2) for d in (-1, 0, 1)}), device="cuda")
    Y, stats, Xp, Yp = torch.empty_like(X), torch.empty(n, 2, device="cuda"), sar.packed_empty(n, K), sar.packed_empty(n, K)
    sar.sar_layernorm_fwd(X, gamma, beta, EPS, Y, stats, Xp, Yp)
    host = lambda p: (p[0][at].cpu().numpy(), p[1][at].cpu().numpy())
    x, st = nw.f64(X[at]), nw.f64(stats[at])
    y, mean, r = nw.norm_fwd(x, nw.f64(gamma), nw.f64(beta), EPS)
    assert np.abs(st - np.concatenate([mean, r], 1)).max() <= 64 * nw.U * 4          # (numbers below 4; 48 roundings and some)
    assert (np.abs(nw.f64(Y[at]) - y) <= nw.half_step(BF16)(np.abs(y)) + 2.0 ** -9 * 2.0 ** -7 + 256 * nw.U * 8).all()
    for p, rows in ((Xp, X), (Yp, Y)):
        q, e = nw.pack(nw.f64(rows[at]))
        assert np.array_equal(host(p)[0], q) and np.array_equal(host(p)[1], e)
    back = torch.empty_like(X)
    sar.sar_unpack(Xp, back)
    assert np.array_equal(nw.f64(back[at]), nw.unpack(*host(Xp), K))
    q, e = sar.packed_empty(n, K)
    sar.sar_pack(X, (q, e))
    assert torch.equal(q, Xp[0]) and torch.equal(e, Xp[1])
    del q, e, back

    ends = [0, 1_000_001, 1_000_001, n - 3]
    W, ptr, work = rn(3, K, F, dtype=F32) / K ** 0.5, torch.tensor(ends, dtype=torch.int32, device="cuda"), work_for(n, K, F, 3)
    Z, dZ, dY = torch.zeros(n, F, dtype=BF16, device="cuda"), rn(n, F), torch.zeros_like(X)
    of = np.searchsorted(ends[1:], at.cpu().numpy(), side="right")
    sar.sar_linear_typed_fwd(Y, W, ptr, Z, work)
    dW = [torch.empty_like(W) for _ in range(2)]
    sar.sar_linear_typed_bwd(Yp, dZ, W, ptr, False, dW[0], dY, work)
    sar.sar_linear_typed_bwd(Y, dZ, W, ptr, False, dW[1], None, work)
    for i, (row, t) in enumerate(zip(at.tolist(), of.tolist())):
        if t < 3:
            rows_close(Z[row:row + 1], nw.f64(Y[row:row + 1]), nw.f64(W[t]), BF16)
            rows_close(dY[row:row + 1], nw.f64(dZ[row:row + 1]), nw.f64(W[t]).T, BF16)
    assert not bool(Z[n - 3:].any()) and not bool(dY[n - 3:].any())
    sums = [torch.zeros(3, K, F, dtype=torch.float64, device="cuda") for _ in range(2)]
    for t, lo, hi in nw.spans(ends, n):
        for a in range(lo, hi, 1 << 18):
            b = min(a + (1 << 18), hi)
            step = torch.exp2(Yp[1][a:b].double() - 127).repeat_interleave(32, 1)
            for s, rows in zip(sums, (Yp[0][a:b].double() * step, Y[a:b].double())):
                s[t] += rows.T.contiguous() @ dZ[a:b].double()
    for got, want in zip(dW, sums):
        for t, lo, hi in nw.spans(ends, n):
            # sums of products of numbers of size 1: roundings of either sign (32 units of sqrt(rows); six times that for the largest of them)
            assert float((got[t].double() - want[t]).abs().max()) <= 6 * 32 * nw.U * max(hi - lo, 1) ** 0.5
    del sums, Z, Yp, Y

    dX, dg, db = torch.empty_like(X), torch.empty(K, device="cuda"), torch.empty(K, device="cuda")
    nwork = torch.empty(sar.sar_layernorm_workspace_bytes(n, K), dtype=torch.uint8, device="cuda")
    for rows in (Xp, X):
        sar.sar_layernorm_bwd(dY, rows, stats, gamma, False, dX, dg, db, nwork)
        x = nw.unpack(*host(Xp), K) if rows is Xp else nw.f64(X[at])
        want, _, _ = nw.norm_bwd(nw.f64(dY[at]), x, st[:, :1], st[:, 1:], nw.f64(gamma))
        assert (np.abs(nw.f64(dX[at]) - want) <= nw.half_step(BF16)(np.abs(want)) + 256 * nw.U * 16).all()
        sg, sb = torch.zeros(K, dtype=torch.float64, device="cuda"), torch.zeros(K, dtype=torch.float64, device="cuda")
        for a in range(0, n, 1 << 18):
            b = min(a + (1 << 18), n)
            v = Xp[0][a:b].double() * torch.exp2(Xp[1][a:b].double() - 127).repeat_interleave(32, 1) if rows is Xp else X[a:b].double()
            d = dY[a:b].double()
            sg += (d * (v - stats[a:b, :1].double()) * stats[a:b, 1:].double()).sum(0)
            sb += d.sum(0)
        # (numbers of size 1, a few thousand roundings behind each other of sums up to sqrt(n))
        assert float((dg.double() - sg).abs().max()) <= 256 * nw.U * n ** 0.5 and float((db.double() - sb).abs().max()) <= 256 * nw.U * n ** 0.5


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,K,F", [(1, 65536, 3), (1, 3, 65536), (70, 65536, 3), (70, 3, 65536), (1500, 65536, 5), (1500, 5, 65536)])
def test_the_widest_weights(n, K, F, dtype):
    g = torch.Generator().manual_seed(n + K)
    X, dZ = torch.randn(n, K, generator=g).to(dtype).cuda(), torch.randn(n, F, generator=g).to(dtype).cuda()
    W = (torch.randn(2, K, F, generator=g) / K ** 0.5).cuda()
    ends = [0, n // 2, n]
    ptr, work = torch.tensor(ends, dtype=torch.int32, device="cuda"), work_for(n, K, F, 2)
    p = sar.packed_empty(n, K)
    sar.sar_pack(X, p)
    Z, dX, dW = torch.empty_like(dZ), torch.empty_like(X), torch.empty_like(W)
    sar.sar_linear_typed_fwd(X, W, ptr, Z, work)
    x, z, w = nw.f64(X), nw.f64(dZ), nw.f64(W)
    for rows in (X, p):
        sar.sar_linear_typed_bwd(rows, dZ, W, ptr, False, dW, dX, work)
        v, got = x if rows is X else nw.unpack(p[0].cpu().numpy(), p[1].cpu().numpy(), K), nw.f64(dW)
        for t, lo, hi in nw.spans(ends, n):
            size = np.abs(v[lo:hi]).T @ np.abs(z[lo:hi])
            assert (np.abs(got[t] - v[lo:hi].T @ z[lo:hi]) <= (64 + (hi - lo) / 32) * 2 * nw.U * size).all()
            if rows is X:
                rows_close(Z[lo:hi], x[lo:hi], w[t], dtype)
                rows_close(dX[lo:hi], z[lo:hi], w[t].T, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [300, 200_000])
def test_the_most_types(n, dtype):
    """65535 of them, most with a few rows or none."""
    T, K, F = 65535, 8, 12
    rng = np.random.default_rng(n)
    of = np.sort(rng.integers(0, T, n))
    ends = np.searchsorted(of, np.arange(T + 1)).astype(np.int32)
    g = torch.Generator().manual_seed(n)
    X, dZ = torch.randn(n, K, generator=g).to(dtype).cuda(), torch.randn(n, F, generator=g).to(dtype).cuda()
    W, ptr, work = torch.randn(T, K, F, generator=g).cuda(), torch.from_numpy(ends).cuda(), work_for(n, K, F, T)
    Z, dX, dW = torch.empty_like(dZ), torch.empty_like(X), torch.empty_like(W)
    sar.sar_linear_typed_fwd(X, W, ptr, Z, work)
    sar.sar_linear_typed_bwd(X, dZ, W, ptr, False, dW, dX, work)
    x, z, w = nw.f64(X), nw.f64(dZ), nw.f64(W)[of]
    for got, want, size, C in ((Z, np.einsum("ik,ikf->if", x, w), np.einsum("ik,ikf->if", np.abs(x), np.abs(w)), K),
                               (dX, np.einsum("if,ikf->ik", z, w), np.einsum("if,ikf->ik", np.abs(z), np.abs(w)), F)):
        off = rows_off(size, C, dtype)
        if dtype == BF16:
            off = off + nw.half_step(dtype)(np.abs(want) + off)
        assert (np.abs(nw.f64(got) - want) <= off).all()
    want, size = np.zeros((T, K, F)), np.zeros((T, K, F))
    np.add.at(want, of, x[:, :, None] * z[:, None, :])
    np.add.at(size, of, np.abs(x[:, :, None] * z[:, None, :]))
    assert (np.abs(nw.f64(dW) - want) <= 130 * nw.U * size).all()
