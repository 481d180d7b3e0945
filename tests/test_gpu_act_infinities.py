"""Infinities and NaN among what the backward pass of the transform with its activation reads: every gradient has what its formula's sum has."""
import pytest
import torch

from tests import nodewise as nw
from tests.test_gpu_act_gradients import run
from tests.test_gpu_linear_act import act, f64, inputs, stored
from tests.test_gpu_linear_typed import dw_off, rows_off

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
INF = float("inf")
ALL = ("dW", "db", "dX", "dA")


def special(t):
    """0: a number, 1: infinity, 2: minus infinity, 3: NaN."""
    return torch.isposinf(t) * 1 + torch.isneginf(t) * 2 + torch.isnan(t) * 3


def same(got, want, tol, what):
    got, want, tol = f64(got).cpu(), want.cpu(), tol.cpu()
    assert torch.equal(special(got), special(want)), what
    fine = torch.isfinite(want)
    assert ((got - want).abs() <= tol)[fine].all(), what


def check(n, K, F, dtype, name, want, in_X, in_dY):
    X, W, _, dY = inputs(n, K, F, dtype, 6)
    A = (2 * torch.randn(n, F, generator=torch.Generator("cuda").manual_seed(n + F), device="cuda")).to(dtype)
    r = [0, n // 2, n - 1]
    if in_X:
        X[r[0], 1], X[r[1], K // 2], X[r[2], K - 1] = INF, -INF, float("nan")
    if in_dY:
        dY[r[0], 0], dY[r[1], F // 2], dY[r[2], F - 1] = INF, -INF, float("nan")
        A[r[0], 0], A[r[1], F // 2] = 1.5, 0.75            # (slopes that are numbers other than zero)
    out = run(X, W, dY, A, name, want)
    x, w, d = f64(X).cpu(), f64(W).cpu(), f64(dY).cpu()
    _, slope, _, off_slope = (t.cpu() for t in act(name, f64(A)))
    off = torch.nan_to_num(d.abs(), 0, 0) * (off_slope + 2 * nw.U * slope.abs())
    # (of ReLU what has no slope has no part, whatever dY holds there)
    d = torch.where(f64(A).cpu() > 0, d, 0.0) if name == "relu" else d * slope
    plain = lambda t: torch.nan_to_num(t, 0, 0, 0).abs()          # (of what is finite: sums with the others are compared by their kind)
    if "dA" in want:
        same(out["dA"], d, stored(dtype, off, plain(d)), "dA")
    if "db" in want:
        same(out["db"], d.sum(0), off.sum(0) + (n / 256 + 64) * 2 * nw.U * plain(d).sum(0), "db")
    if "dW" in want:
        size = plain(x).T @ plain(d)
        same(out["dW"], x.T @ d, plain(x).T @ off + 2 * dw_off(size, n) + 2.0 ** -17 * size, "dW")
    if "dX" in want:
        size, exact = plain(d) @ w.abs().T, d @ w.T
        tol = off @ w.abs().T + rows_off(size, 2 * F, dtype) + (2.0 ** -17 + 2.0 ** -16) * size
        same(out["dX"], exact, stored(dtype, tol, plain(exact)), "dX")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("name", ["none", "relu", "silu"])
# few rows, few rows of which dX has many columns, many, kept operands, more than what is kept
@pytest.mark.parametrize("n,K,F", [(300, 40, 72), (100, 40_000, 32), (2000, 64, 128), (3000, 40, 71), (20_000, 300, 260), (65_600, 80, 72), (65_600, 80, 255)])
def test_they_reach_the_gradients_that_have_them(n, K, F, name, dtype):
    for in_X, in_dY in ((True, False), (False, True), (True, True)):
        check(n, K, F, dtype, name, ALL, in_X, in_dY)
        check(n, K, F, dtype, name, ("dW", "db"), in_X, in_dY)
        check(n, K, F, dtype, name, ("dW", "dX"), in_X, in_dY)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("name", ["none", "relu", "silu"])
@pytest.mark.parametrize("n,K,F", [(300, 40, 72), (100, 40_000, 32), (3000, 40, 71), (65_600, 80, 72)])
def test_without_the_rows_gradient(n, K, F, name, dtype):
    for in_X, in_dY in ((False, False), (True, False), (False, True)):
        check(n, K, F, dtype, name, ("dW", "dA"), in_X, in_dY)
        check(n, K, F, dtype, name, ("dW", "db", "dA"), in_X, in_dY)
