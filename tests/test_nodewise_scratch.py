"""How much scratch the node-wise calls ask for, and what they do with it."""
import pytest
import torch

from paper_2111_06483_amd import sar

SHAPES = [(1, 1), (47, 200), (64, 64), (100, 47), (128, 128), (100, 256), (200, 47), (256, 100), (256, 256), (400, 400), (512, 512), (1024, 96)]


def row_counts():
    """Around the multiples of 32 rows and of the powers of two, where the numbers of workgroups change, and between them."""
    some = {n + d for k in range(5, 21) for n in (1 << k, 3 << (k - 1)) for d in (-1, 0, 1, 31, 32, 33)}
    return sorted(some | set(range(0, 400)) | set(range(400, 40_000, 97)) | set(range(6100, 6200)) | set(range(24_500, 24_600)))


@pytest.mark.parametrize("T", [1, 4, 37])
@pytest.mark.parametrize("K,F", SHAPES)
def test_scratch_of_a_larger_batch_serves_a_smaller_one(K, F, T):
    """A program asks once, for the most rows it has."""
    least = 0
    for n in row_counts():
        size = sar.sar_linear_typed_workspace_bytes(n, K, F, T)
        assert size >= least, n
        least = size


@pytest.mark.parametrize("D", [1, 8, 47, 64, 256, 1000, 1025, 4096, 8192])
def test_scratch_of_layer_norm_grows_with_the_rows(D):
    sizes = [sar.sar_layernorm_workspace_bytes(n, D) for n in row_counts()]
    assert sizes == sorted(sizes)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,packed", [(torch.float32, False), (torch.float32, True), (torch.bfloat16, False), (torch.bfloat16, True)])
@pytest.mark.parametrize("n,K,F", [(6144, 256, 256), (24_576, 128, 128), (16_000, 100, 47)])
def test_a_batch_in_the_scratch_of_one_more_row(n, K, F, dtype, packed):
    """The same results as in scratch of its own size; nothing behind either is written."""
    from tests import nodewise as nw
    g = torch.Generator().manual_seed(n)
    X, dZ = torch.randn(n, K, generator=g).to(dtype).cuda(), torch.randn(n, F, generator=g).to(dtype).cuda()
    W, ptr = torch.randn(4, K, F, generator=g).cuda(), torch.tensor([0, n // 5, n // 2, n // 2, n], dtype=torch.int32, device="cuda")
    rows = X
    if packed:
        rows = sar.packed_empty(n, K)
        sar.sar_pack(X, rows)
    got = []
    for more in (0, 1):
        size = sar.sar_linear_typed_workspace_bytes(n + more, K, F, 4)
        room = torch.full((size + 4096,), 77, dtype=torch.uint8, device="cuda")
        Z, dW, dX = torch.empty_like(dZ), torch.empty_like(W), torch.empty_like(X)
        sar.sar_linear_typed_fwd(X, W, ptr, Z, room[:size])
        sar.sar_linear_typed_bwd(rows, dZ, W, ptr, False, dW, dX, room[:size])
        assert bool((room[size:] == 77).all())
        got.append((Z, dW, dX))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    x = nw.f64(X) if not packed else nw.unpack(rows[0].cpu().numpy(), rows[1].cpu().numpy(), K)
    for t, lo, hi in nw.spans(ptr.tolist(), n):
        d = nw.f64(dZ[lo:hi])
        # (as many roundings of a sum as it has chunks of 32 rows, and the workgroups')
        assert (abs(nw.f64(got[0][1][t]) - x[lo:hi].T @ d) <= (64 + (hi - lo) / 32) * 2 * nw.U * (abs(x[lo:hi]).T @ abs(d))).all()
