"""The backward pass of the transform with its activation: how many bits its gradients keep, in every way they are formed."""
import pytest
import torch

from paper_2111_06483_amd import sar
from tests import nodewise as nw
from tests.test_gpu_linear_act import ACTS, act, check_bwd, f64, inputs, scratch, stored
from tests.test_gpu_linear_typed import rows_off

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DTYPES = [F32, BF16]


def gradients(n, K, F, dtype, name, want, seed=0, accumulate=False):
    """(X, W, dY, A of a call, its outputs)."""
    X, W, _, dY = inputs(n, K, F, dtype, seed)
    g = torch.Generator("cuda").manual_seed(n + F)
    A = (2 * torch.randn(n, F, generator=g, device="cuda")).to(dtype)
    return X, W, dY, A, run(X, W, dY, A, name, want, accumulate)


def run(X, W, dY, A, name, want, accumulate=False):
    (n, F), K, dtype = dY.shape, W.shape[0], dY.dtype
    e = lambda *s, dt=F32: torch.full(s, 3.0, dtype=dt, device="cuda")
    out = {"dW": e(K, F), "db": e(F), "dX": e(n, K, dt=dtype), "dA": e(n, F, dt=dtype)}
    out = {k: v if k in want else None for k, v in out.items()}
    work, behind = scratch(n, K, F)
    sar.sar_linear_act_bwd(dY, A, X if "dW" in want else None, W, ACTS[name], accumulate, out["dW"], out["db"], out["dX"], out["dA"], work)
    assert bool((behind == 77).all())
    return out


# few rows in one launch; few blocks of dX alone; kept operands, whole and ragged; contractions that are not kept; few columns
@pytest.mark.parametrize("want", [("dX",), ("dX", "dA"), ("db", "dX"), ("dW", "dX"), ("dW", "db", "dX", "dA")])
@pytest.mark.parametrize("n,K,F", [(1, 5, 3), (37, 33, 47), (300, 100, 256), (900, 400, 31), (2000, 64, 128), (9001, 200, 400), (30_011, 172, 47), (66_000, 256, 256),
                                   (66_001, 100, 72), (66_005, 72, 47), (66_000, 100, 46), (65_999, 128, 63), (65_999, 128, 127), (66_000, 40, 72), (66_000, 256, 400), (66_000, 129, 260)])
def test_dx_rounds_once(n, K, F, want):
    """bf16: dX = dA W^T from dA = dY act'(A) to 16 bits (two pieces of 8: 2^-17 of it), and what a product of both operands' second pieces is (2^-16
    of a term), rounded once when it is stored; twice as many products are added up."""
    for name in ("gelu", "relu"):
        X, W, dY, A, out = gradients(n, K, F, BF16, name, want)
        _, slope, _, off_slope = act(name, f64(A))
        d, w = f64(dY), f64(W)
        off = d.abs() * (off_slope + 2 * nw.U * slope.abs())
        d = d * slope
        size, exact = d.abs() @ w.abs().T, d @ w.T
        tol = off @ w.abs().T + rows_off(size, 2 * F, BF16) + (2.0 ** -17 + 2.0 ** -16) * size
        assert ((f64(out["dX"]) - exact).abs() <= stored(BF16, tol, exact)).all(), name
        if "dA" in want:
            assert ((f64(out["dA"]) - d).abs() <= stored(BF16, off, d)).all(), name


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("want", [("dW", "dA"), ("db", "dA"), ("dW", "db", "dA"), ("db", "dX", "dA"), ("dW", "db", "dX")])
# few rows; few of which dX has many columns; dX's blocks few and dW's rows not; many
@pytest.mark.parametrize("n,K,F", [(1, 7, 9), (300, 40, 72), (100, 40_000, 32), (2000, 64, 128), (9001, 47, 71), (66_000, 80, 72)])
def test_more_forms(n, K, F, want, dtype):
    for name in ("none", "gelu"):
        check_bwd(n, K, F, dtype, name, want=want, seed=3)
        check_bwd(n, K, F, dtype, name, accumulate=True, want=want, seed=4)
