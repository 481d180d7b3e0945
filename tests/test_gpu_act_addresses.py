"""The gradient of a residual inside the activation at any address: the memory before and behind it stays as it is."""
import pytest
import torch

from paper_2111_06483_amd import sar
from tests.test_gpu_linear_act import ACTS, inputs, scratch
from tests.test_gpu_student_step import moved

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("by", [1, 3])
@pytest.mark.parametrize("want", [("dW", "db", "dX"), ("dW", "db"), ("dX",), ()])
# few rows; ragged rows and widths, even and odd, of every way in which dA is written; last chunks that are not full
@pytest.mark.parametrize("n,K,F", [(301, 33, 46), (900, 70, 31), (2001, 64, 128), (9001, 100, 74), (66_001, 47, 72), (66_001, 100, 72), (65_999, 130, 70), (66_003, 200, 132),
                                   (66_005, 72, 47), (66_007, 129, 258)])
def test_error_rows_at_any_address(n, K, F, want, by, dtype):
    X, W, _, dY = inputs(n, K, F, dtype, 8)
    A = (2 * torch.randn(n, F, generator=torch.Generator("cuda").manual_seed(n), device="cuda")).to(dtype)
    got = []
    for shift in (0, by):
        put = lambda t: moved(t, shift)
        of = {"dW": put(torch.zeros_like(W)), "db": put(torch.zeros(F, device="cuda")), "dX": put(torch.zeros_like(X)), "dA": put(torch.zeros_like(dY))}
        given = {k: of[k][0] if k in want + ("dA",) else None for k in of}
        rows = [put(t)[0] for t in (dY, A, X, W)]
        sar.sar_linear_act_bwd(rows[0], rows[1], rows[2], rows[3], ACTS["silu"], False, given["dW"], given["db"], given["dX"], given["dA"], scratch(n, K, F)[0])
        for k, (t, room) in of.items():
            assert bool((room[:shift] == 77).all()) and bool((room[shift + t.numel():] == 77).all()), k
        got.append({k: t for k, t in given.items() if t is not None})
    for k in got[0]:
        assert torch.equal(got[0][k], got[1][k]), k
    assert bool((got[1]["dA"] != 0).any())
