"""GELU far below zero, where the normal distribution's share is small: how far it is off, relative to itself."""
import math

import pytest
import torch

from paper_2111_06483_amd import sar
from tests import nodewise as nw
from tests.test_gpu_linear_act import ACTS, f64, scratch

pytestmark = pytest.mark.gpu
# The fitted polynomial's own error, relative to the share, up to these distances below zero (in 64 bits, on 20001 points of each interval).
FIT = [(1, 3.6e-8), (2, 1.6e-7), (3, 3.3e-6), (4, 5.1e-5), (5, 2.1e-4), (6, 5.1e-4), (8, 1.7e-3), (10, 3.4e-3), (12, 7.7e-3)]


def test_gelu_far_below_zero():
    a = torch.linspace(-12, 0, 24_001).cuda()
    X = torch.stack([a, torch.zeros_like(a)], 1)
    W = torch.eye(2, device="cuda")
    n = len(a)
    Y, D, work = torch.empty_like(X), torch.empty_like(X), scratch(n, 2, 2)[0]
    sar.sar_linear_act_fwd(X, W, None, None, ACTS["gelu"], False, Y, None, work)
    sar.sar_linear_act_bwd(torch.ones_like(X), X, None, W, ACTS["gelu"], False, None, None, None, D, work)
    x = f64(X)[:, 0]
    share, bell = 0.5 * torch.special.erfc(-x / math.sqrt(2)), torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    fit = torch.zeros_like(x)
    for upto, off in reversed(FIT):
        fit = torch.where(x >= -upto, off, fit)
    # the exponential's argument is rounded three times, each by a unit of it; some 40 units for the polynomial, whose terms have both signs, and the rest
    ops = (2 * x * x + 40) * nw.U
    # (the argument itself arrives through a product: a unit)
    moves = 2 * nw.U * x.abs() * bell * x.abs()
    assert ((f64(Y)[:, 0] - x * share).abs() <= x.abs() * share * (fit + ops) + moves).all()
    assert ((f64(D)[:, 0] - share - x * bell).abs() <= share * (fit + ops) + x.abs() * bell * ops).all()
