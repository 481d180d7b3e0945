"""Layer norm of rows whose values lie far from zero for how far they lie apart, against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2111_06483_amd import sar
from tests import nodewise as nw

pytestmark = pytest.mark.gpu
EPS = 1e-5
WIDTHS = [3, 47, 100, 200, 256, 777, 1025, 2049, 8191]
CENTRES = [1 / 3, -0.7, 3.3, 255.7, -12345.6, 7.1e6]


def terms(D):
    """Additions behind a sum over a row: a lane's values one after the other, the lanes by halves; a few more operations."""
    return min(D, 32) + 16


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", WIDTHS)
def test_constant_rows_are_beta(D, dtype):
    """A first mean is a few units in its last place off; the mean of the deviations from it, added, leaves the value itself: that the deviations are
    c - mean is exact, and their mean is off by 48 roundings of a number that is 48 units of c at most, 2^-36 c."""
    X = torch.tensor(CENTRES)[:, None].expand(-1, D).contiguous().to(dtype).cuda()
    gamma, beta = torch.full((D,), 2.0, device="cuda"), torch.randn(D, generator=torch.Generator().manual_seed(D)).cuda()
    Y, stats = torch.empty_like(X), torch.empty(len(CENTRES), 2, device="cuda")
    sar.sar_layernorm_fwd(X, gamma, beta, EPS, Y, stats)
    assert torch.equal(stats[:, 0], X[:, 0].float())
    r = 1 / np.sqrt(np.float64(np.float32(EPS)))
    assert (np.abs(nw.f64(stats[:, 1]) - r) <= 4 * nw.U * r).all()
    assert torch.equal(Y, beta.to(dtype).expand_as(Y))


@pytest.mark.parametrize("spread", [1e-3, 1.0])
@pytest.mark.parametrize("D", WIDTHS)
def test_rows_far_from_zero(D, spread):
    """The mean is off by its own rounding and little else; the deviations' sum being zero, an error of the mean enters the variance squared."""
    g = torch.Generator().manual_seed(D)
    X = (torch.tensor(CENTRES)[:, None] + spread * torch.randn(len(CENTRES), D, generator=g)).cuda()
    x = nw.f64(X)
    Y, stats = torch.empty_like(X), torch.empty(len(CENTRES), 2, device="cuda")
    sar.sar_layernorm_fwd(X, None, None, EPS, Y, stats)
    y, mean, r = nw.norm_fwd(x, 1.0, 0.0, np.float64(np.float32(EPS)))
    s = nw.f64(stats)
    # the deviations from a first mean are at most `spread`'s scale and that mean's error; they are rounded, and so is their sum, terms(D) times
    dev = np.abs(x - mean).mean(1, keepdims=True) + terms(D) * nw.U * np.abs(x).mean(1, keepdims=True)
    off_mean = nw.U * np.abs(mean) + (terms(D) + 4) * nw.U * dev
    off_r = r * ((terms(D) + 8) * nw.U + (off_mean * r) ** 2)
    assert (np.abs(s[:, :1] - mean) <= off_mean).all()
    assert (np.abs(s[:, 1:] - r) <= off_r).all()
    assert (np.abs(nw.f64(Y) - y) <= off_mean * r + np.abs(x - mean) * (off_r + 4 * nw.U * r)).all()
