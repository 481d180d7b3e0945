"""Backward passes of many rows in every way that dA takes: the same bits every time, on two streams at once and replayed from graphs."""
import pytest
import torch

from paper_2111_06483_amd import sar
from tests.test_gpu_linear_act import ACTS, inputs, scratch

pytestmark = pytest.mark.gpu
# few rows in one launch; few rows, dX of many columns; dX's blocks few; dX by tiles; one kept block of columns; two; rows that are not whole words
SHAPES = [(300, 40, 72), (100, 40_000, 32), (2000, 64, 128), (20_000, 300, 140), (66_001, 100, 72), (66_000, 132, 72), (66_003, 200, 95)]


class Pass:
    def __init__(self, n, K, F, dtype, seed):
        self.X, self.W, _, self.dY = inputs(n, K, F, dtype, seed)
        self.A = (2 * torch.randn(n, F, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")).to(dtype)
        self.out = [torch.zeros_like(self.W), torch.zeros(F, device="cuda"), torch.zeros_like(self.X), torch.zeros_like(self.dY)]
        self.work = scratch(n, K, F)[0]

    def run(self, rows=True):
        sar.sar_linear_act_bwd(self.dY, self.A, self.X, self.W, ACTS["gelu"], False, self.out[0], self.out[1], self.out[2], self.out[3] if rows else None, self.work)

    def results(self):
        return [t.clone() for t in self.out]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [True, False])
@pytest.mark.parametrize("n,K,F", SHAPES)
def test_the_same_bits(n, K, F, rows, dtype):
    passes = [Pass(n, K, F, dtype, seed) for seed in (1, 2)]
    want = []
    for p in passes:
        p.run(rows)
        want.append(p.results())
        p.work.fill_(0xff)                     # (nothing of a call is left for the next one)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in passes]
    for _ in range(4):
        for p, st in zip(passes, streams):
            with torch.cuda.stream(st):
                p.run(rows)
    torch.cuda.synchronize()
    for p, w in zip(passes, want):
        assert all(torch.equal(a, b) for a, b in zip(p.results(), w))
    graphs = []
    for p in passes:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            p.run(rows)
        graphs.append(g)
    for turn in range(3):
        for p, g in zip(passes, graphs):
            p.dY.mul_(0.5)
            for t in p.out:
                t.zero_()
            p.work.fill_(0xff)
            g.replay()
            torch.cuda.synchronize()
            got = p.results()
            p.run(rows)
            assert all(torch.equal(a, b) for a, b in zip(got, p.results())), turn
