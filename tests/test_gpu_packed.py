"""Rows in 8 bits against their definition, byte by byte."""
import numpy as np
import pytest
import torch

from paper_2111_06483_amd import sar
from tests import nodewise as nw

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16]


def guarded(n, width, dtype):
    """A tensor with 64 values before and behind it that nobody may write."""
    fill = 77
    buf = torch.full((n * width + 128,), fill, dtype=dtype, device="cuda")
    return buf, buf[64:64 + n * width].view(n, width)


def untouched(buf):
    return bool((buf[:64] == 77).all()) and bool((buf[-64:] == 77).all())


def check(X):
    n, K = X.shape
    qb, q = guarded(n, -(-K // 16) * 16, torch.int8)
    eb, e = guarded(n, -(-K // 32), torch.uint8)
    sar.sar_pack(X, (q, e))
    want_q, want_e = nw.pack(nw.f64(X))
    assert (e.cpu().numpy() == want_e).all()
    assert (q.cpu().numpy() == want_q).all()
    assert untouched(qb) and untouched(eb)
    for dt in DTYPES:
        bb, back = guarded(n, K, dt)
        sar.sar_unpack((q, e), back)
        got, want = nw.f64(back), nw.unpack(want_q, want_e, K)
        assert np.array_equal(got, want, equal_nan=True)
        assert untouched(bb)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 47, 64, 95, 100, 130, 257, 1030])
@pytest.mark.parametrize("n", [1, 3, 130])
def test_rows_of_every_width(n, K, dtype):
    g = torch.Generator().manual_seed(K * 1000 + n)
    X = (torch.randn(n, K, generator=g) * torch.exp2(torch.randint(-40, 40, (n, 1), generator=g).float())).to(dtype).cuda()
    check(X)


@pytest.mark.parametrize("dtype", DTYPES)
def test_more_rows_than_a_workgroup_has_units_for(dtype):
    g = torch.Generator().manual_seed(1)
    check(torch.randn(5003, 100, generator=g).to(dtype).cuda())
    check(torch.randn(20011, 7, generator=g).to(dtype).cuda())


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_that_begin_anywhere(dtype):
    g = torch.Generator().manual_seed(2)
    buf = torch.randn(40 * 47 + 1, generator=g).to(dtype).cuda()
    check(buf[1:].view(40, 47))


@pytest.mark.parametrize("dtype", DTYPES)
def test_values_at_the_borders(dtype):
    big = float(torch.finfo(dtype).max)
    tiny = 2.0 ** -149 if dtype == torch.float32 else 2.0 ** -133
    rows = [[0.0], [-0.0, 0.0], [127.0, -127.0], [127.5, 1.0], [-127.5, 0.5], [127.0, 0.5, 1.5, 2.5, -0.5, -1.5], [128.0, 1.0, 3.0],
            [255.0, 1.0], [254.0, 1.0, 3.0], [big, -big, 1.0], [tiny, -tiny], [2.0 ** -126, tiny, 2.0 ** -127, -3 * 2.0 ** -127],
            [2.0 ** -120, 2.0 ** -127], [2.0 ** -119, 2.0 ** -127], [float("inf"), 1.0], [1.0, float("nan")], [-float("inf")],
            [1e-30, 1e-32], [1.9921875, 0.0078125], [1.984375, 0.0078125]]
    X = torch.zeros(len(rows), 70)
    for i, r in enumerate(rows):
        X[i, 33:33 + len(r)] = torch.tensor(r)                   # the blocks beside it are zero
    check(X.to(dtype).cuda())


def test_no_rows():
    q, e = sar.packed_empty(0, 40)
    sar.sar_pack(torch.empty(0, 40, device="cuda"), (q, e))
    sar.sar_unpack((q, e), torch.empty(0, 40, device="cuda"))


def test_offsets_beyond_32_bits():
    """2^32 bytes of numbers and more: the last rows of a tall bf16 tensor."""
    n, K = (1 << 25) + 5, 144
    X = torch.zeros(n, K, dtype=torch.bfloat16, device="cuda")
    X[-3:] = torch.randn(3, K, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
    p = sar.packed_empty(n, K)
    sar.sar_pack(X, p)
    want_q, want_e = nw.pack(nw.f64(X[-3:]))
    assert (p[0][-3:].cpu().numpy() == want_q).all() and (p[1][-3:].cpu().numpy() == want_e).all()
    last = X[-3:].clone()
    X.fill_(7)
    sar.sar_unpack(p, X)
    assert np.array_equal(nw.f64(X[-3:]), nw.unpack(want_q, want_e, K))
    assert bool((X[:-3] == 0).all()) and last.shape == (3, K)
