"""The forward pass of the transform with its epilogue needs the scratch of a typed transform alone, not what the backward pass keeps of its rows."""
import pytest
import torch

from paper_2111_06483_amd import sar
from tests.test_gpu_linear_act import inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
# few rows; tiles of two, four and eight columns' tiles; kept operands
@pytest.mark.parametrize("n,K,F", [(300, 40, 72), (20_011, 130, 47), (30_000, 300, 128), (40_001, 513, 257), (66_001, 100, 256)])
def test_the_scratch_of_the_forward_pass(n, K, F, dtype):
    X, W, b, R = inputs(n, K, F, dtype)
    size = sar.sar_linear_typed_workspace_bytes(n, K, F, 1)
    assert size < sar.sar_linear_act_workspace_bytes(n, K, F)
    room = torch.full((size + 4096,), 77, dtype=torch.uint8, device="cuda")
    much = torch.empty(sar.sar_linear_act_workspace_bytes(n, K, F), dtype=torch.uint8, device="cuda")
    got = []
    for work in (room[:size], much):
        Y, A = torch.empty_like(R), torch.empty_like(R)
        sar.sar_linear_act_fwd(X, W, b, R, sar.SAR_ACT_GELU, False, Y, A, work)
        got += [Y, A]
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3])
    assert bool((room[size:] == 77).all())
