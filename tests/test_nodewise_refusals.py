"""What the node-wise calls refuse, before anything reaches a device (tensors in host memory serve for that)."""
import ctypes

import pytest
import torch

from paper_2111_06483_amd import sar

F32, BF16 = torch.float32, torch.bfloat16
i64 = ctypes.c_int64


@pytest.fixture(scope="module", autouse=True)
def built():
    sar.native()


def refused(call, text, code=sar.SAR_ERR_INVALID_ARG):
    with pytest.raises(sar.SarError) as e:
        call()
    assert e.value.code == code and text in str(e.value), str(e.value)


def t(*shape, dtype=F32):
    return torch.zeros(*shape, dtype=dtype)


def host_packed(n, K):
    return sar.packed_empty(n, K, device="cpu")


def test_tensors_in_host_memory():
    p, w = host_packed(4, 8), t(1024, dtype=torch.uint8)
    ptr = t(3, dtype=torch.int32)
    for call in (lambda: sar.sar_pack(t(4, 8), p), lambda: sar.sar_unpack(p, t(4, 8)),
                 lambda: sar.sar_layernorm_fwd(t(4, 8), t(8), t(8), 1e-5, t(4, 8), t(4, 2), p, p),
                 lambda: sar.sar_layernorm_bwd(t(4, 8), t(4, 8), t(4, 2), t(8), False, t(4, 8), t(8), t(8), w),
                 lambda: sar.sar_layernorm_bwd(t(4, 8), p, t(4, 2), None, False, t(4, 8), None, None, None),
                 lambda: sar.sar_linear_typed_fwd(t(4, 8), t(2, 8, 6), ptr, t(4, 6), w),
                 lambda: sar.sar_linear_typed_bwd(t(4, 8), t(4, 6), t(2, 8, 6), ptr, False, t(2, 8, 6), t(4, 8), w),
                 lambda: sar.sar_linear_bwd_packed(p, t(4, 6), t(8, 6), False, t(8, 6), t(4, 8), w)):
        refused(call, "host memory")


def test_shapes_that_do_not_fit():
    p, w, ptr = host_packed(4, 8), t(1024, dtype=torch.uint8), t(3, dtype=torch.int32)
    X, dY = t(4, 8), t(4, 8)
    norm = lambda **k: sar.sar_layernorm_fwd(*{**dict(X=X, gamma=t(8), beta=t(8), eps=1e-5, Y=t(4, 8), stats=t(4, 2), Xp=None, Yp=None), **k}.values())
    refused(lambda: norm(gamma=t(7)), "gamma has shape (7,), the call needs (8)")
    refused(lambda: norm(beta=t(8, 1)), "beta")
    refused(lambda: norm(Y=t(5, 8)), "Y has shape")
    refused(lambda: norm(stats=t(4)), "stats")
    refused(lambda: norm(Xp=host_packed(3, 8)), "Xp")
    refused(lambda: norm(Yp=host_packed(4, 40)), "Yp")
    refused(lambda: norm(Yp=(p[0],)), "a pair (q, e)")
    back = lambda **k: sar.sar_layernorm_bwd(*{**dict(dY=dY, X=X, stats=t(4, 2), gamma=t(8), accumulate=False, dX=t(4, 8), dgamma=t(8), dbeta=t(8), work=w), **k}.values())
    refused(lambda: back(X=t(4, 9)), "X has shape")
    refused(lambda: back(X=host_packed(5, 8)), "X has shape")
    refused(lambda: back(stats=t(8)), "stats")
    refused(lambda: back(dX=t(8, 4)), "dX")
    refused(lambda: back(dgamma=t(9)), "dgamma")
    refused(lambda: back(dbeta=t(1, 8)), "dbeta")
    fwd = lambda **k: sar.sar_linear_typed_fwd(*{**dict(X=X, W=t(2, 8, 6), ptr=ptr, Z=t(4, 6), work=w), **k}.values())
    refused(lambda: fwd(W=t(2, 7, 6)), "W has shape")
    refused(lambda: fwd(ptr=t(2, dtype=torch.int32)), "type_ptr has shape")
    refused(lambda: fwd(Z=t(4, 7)), "Z has shape")
    bwd = lambda **k: sar.sar_linear_typed_bwd(*{**dict(X=X, dZ=t(4, 6), W=t(2, 8, 6), ptr=ptr, acc=False, dW=t(2, 8, 6), dX=t(4, 8), work=w), **k}.values())
    refused(lambda: bwd(X=t(3, 8)), "X has shape")
    refused(lambda: bwd(dZ=t(4, 5)), "W has shape")
    refused(lambda: bwd(dW=t(8, 6)), "dW has shape")
    refused(lambda: bwd(dX=t(4, 6)), "dX has shape")
    one = lambda **k: sar.sar_linear_bwd_packed(*{**dict(p=p, dZ=t(4, 6), W=t(8, 6), acc=False, dW=t(8, 6), dX=t(4, 8), work=w), **k}.values())
    refused(lambda: one(p=host_packed(4, 17)), "X has shape")
    refused(lambda: one(W=t(8, 7)), "W has shape")
    refused(lambda: sar.sar_pack(X, None), "a pair (q, e)")
    refused(lambda: sar.sar_unpack(None, X), "a pair (q, e)")
    with pytest.raises(ValueError):
        sar.sar_pack(t(8), p)
    with pytest.raises(ValueError):
        fwd(W=t(8, 6))


def test_types_that_do_not_fit():
    p, w = host_packed(4, 8), t(1024, dtype=torch.uint8)
    refused(lambda: sar.sar_pack(t(4, 8, dtype=torch.float16), p), "torch.float16", sar.SAR_ERR_UNSUPPORTED)
    refused(lambda: sar.sar_pack(t(4, 8), (p[0].float(), p[1])), "torch.int8")
    refused(lambda: sar.sar_pack(t(4, 8), (p[0], p[1].to(torch.int8))), "torch.uint8")
    refused(lambda: sar.sar_layernorm_fwd(t(4, 8), t(8, dtype=BF16), None, 1e-5, t(4, 8)), "gamma is torch.bfloat16")
    refused(lambda: sar.sar_layernorm_fwd(t(4, 8), None, None, 1e-5, t(4, 8, dtype=BF16)), "Y is torch.bfloat16")
    refused(lambda: sar.sar_layernorm_bwd(t(4, 8, dtype=BF16), t(4, 8), t(4, 2), None, False, None, t(8), t(8), w), "X is torch.float32")
    refused(lambda: sar.sar_linear_typed_fwd(t(4, 8), t(2, 8, 6), t(3, dtype=torch.int64), t(4, 6), w), "type_ptr is torch.int64")
    refused(lambda: sar.sar_linear_typed_fwd(t(4, 8), t(2, 8, 6, dtype=BF16), t(3, dtype=torch.int32), t(4, 6), w), "W is torch.bfloat16")
    refused(lambda: sar.sar_linear_bwd_packed(p, t(4, 6), t(8, 6), False, t(8, 6, dtype=BF16), None, w), "dW is torch.bfloat16")


def test_tensors_that_are_no_plain_memory():
    p, w = host_packed(4, 8), t(1024, dtype=torch.uint8)
    refused(lambda: sar.sar_pack(t(8, 4).T, p), "X must be contiguous")
    refused(lambda: sar.sar_layernorm_fwd(t(4, 8), t(16)[::2], None, 1e-5, t(4, 8)), "gamma must be contiguous")
    refused(lambda: sar.sar_layernorm_fwd(t(4, 8), None, None, 1e-5, t(4, 16)[:, ::2]), "Y must be contiguous")
    refused(lambda: sar.sar_linear_typed_fwd(t(4, 8), t(2, 6, 8).transpose(1, 2), t(3, dtype=torch.int32), t(4, 6), w), "W must be contiguous")
    for call in (lambda: sar.sar_pack(None, p), lambda: sar.sar_layernorm_fwd(None, None, None, 1e-5, t(4, 8)),
                 lambda: sar.sar_layernorm_fwd(t(4, 8), None, None, 1e-5, None), lambda: sar.sar_linear_typed_fwd(t(4, 8), None, None, None, w)):
        with pytest.raises(AttributeError):
            call()


def test_errors_of_the_library():
    lib, none = sar.lib(), None
    n = ctypes.c_size_t()
    err = lambda: lib.sar_last_error().decode()
    some = ctypes.create_string_buffer(4096)
    at = (ctypes.addressof(some) + 255) // 256 * 256                # (never read: the calls are refused first)
    bad, unsupported = sar.SAR_ERR_INVALID_ARG, sar.SAR_ERR_UNSUPPORTED
    # rows in 8 bits
    assert lib.sar_pack(none, 0, 4, 8, none, none, none) == bad and "null" in err()
    assert lib.sar_pack(at, 2, 4, 8, at, at, none) == unsupported
    assert lib.sar_pack(at, 0, -1, 8, at, at, none) == bad
    assert lib.sar_pack(at, 0, 4, 0, at, at, none) == bad
    assert lib.sar_pack(at, 0, 4, (1 << 24) + 1, at, at, none) == unsupported
    assert lib.sar_pack(at, 0, 4, 8, at + 8, at, none) == bad and "16-byte" in err()
    assert lib.sar_unpack(at, none, 0, 4, 8, at, none) == bad
    assert lib.sar_pack(none, 0, 0, 8, none, none, none) == 0
    # layer norm
    fwd = lambda X=at, eps=1e-5, Y=at, dt=0, rows=4, D=8, xq=none, xe=none: lib.sar_layernorm_fwd(X, none, none, eps, Y, none, dt, rows, D, xq, xe, none, none, none)
    assert fwd(X=none) == bad and "null" in err()
    assert fwd(Y=none) == bad
    assert fwd(eps=-1.0) == bad and "eps" in err()
    assert fwd(eps=float("nan")) == bad
    assert fwd(dt=5) == unsupported
    assert fwd(D=0) == bad
    assert fwd(D=8193) == unsupported and "8192" in err()
    assert fwd(rows=-1) == bad
    assert fwd(xq=at) == bad and "both" in err()
    assert fwd(xq=at + 4, xe=at) == bad and "16-byte" in err()
    assert fwd(X=none, Y=none, rows=0) == 0
    bwd = lambda dY=at, X=at, xq=none, xe=none, stats=at, dX=at, dg=at, rows=4000, work=at, size=1 << 40: lib.sar_layernorm_bwd(
        dY, X, xq, xe, stats, none, 0, dX, dg, none, 0, rows, 8, work, size, none)
    assert bwd(dY=none) == bad and bwd(X=none) == bad and bwd(stats=none) == bad
    assert bwd(xq=at, xe=at) == bad and "both given" in err()
    assert bwd(work=none) == bad and "work" in err()
    assert bwd(size=16) == bad and "needs" in err()
    assert bwd(work=at + 4) == bad and "16-byte" in err()
    assert bwd(dX=none, dg=none, work=none) == 0                      # nothing asked for
    assert lib.sar_layernorm_workspace_bytes(100, 8, ctypes.byref(n)) == 0 and n.value > 0
    assert lib.sar_layernorm_workspace_bytes(100, 9000, ctypes.byref(n)) == unsupported
    assert lib.sar_layernorm_workspace_bytes(100, 8, none) == bad
    # transforms by type
    assert lib.sar_linear_typed_workspace_bytes(1000, 8, 6, 2, ctypes.byref(n)) == 0 and n.value > 0
    size = n.value
    fwd = lambda X=at, W=at, ptr=at, T=2, Z=at + 2048, dt=0, rows=1000, K=8, F=6, work=at, wb=size: lib.sar_linear_typed_fwd(
        X, W, ptr, T, Z, dt, rows, K, F, work, wb, none)
    assert fwd(X=none) == bad and fwd(W=none) == bad and fwd(Z=none) == bad
    assert fwd(Z=at) == bad and "alias" in err()
    assert fwd(ptr=none) == bad and "type_ptr" in err()
    assert fwd(T=0) == bad and fwd(K=0) == bad and fwd(F=0) == bad and fwd(rows=-1) == bad
    assert fwd(T=65536) == unsupported and fwd(K=65537) == unsupported and fwd(rows=1 << 31) == unsupported and fwd(dt=3) == unsupported
    assert fwd(work=none) == bad and fwd(wb=size - 1) == bad and fwd(work=at + 8) == bad
    bwd = lambda X=at, xq=none, xe=none, dZ=at, W=at, dW=at, dX=at + 2048, wb=size: lib.sar_linear_typed_bwd(
        X, xq, xe, dZ, W, at, 2, 0, dW, dX, 0, 1000, 8, 6, at, wb, none)
    assert bwd(dZ=none) == bad and bwd(X=none) == bad and bwd(W=none) == bad
    assert bwd(xq=at, xe=at) == bad and "both given" in err()
    assert bwd(X=none, xq=at) == bad and bwd(X=none, xq=at + 8, xe=at) == bad
    assert bwd(dX=at) == bad and "alias" in err()
    assert bwd() == bad and "dW must not alias W" in err()
    assert bwd(wb=0) == bad
    assert bwd(dW=none, dX=none) == 0
    assert lib.sar_linear_bwd_packed(none, none, at, at, 0, at, none, 0, 1000, 8, 6, at, 1 << 40, none) == bad
    assert lib.sar_linear_bwd_packed(at, at, at, at, 0, at, none, 0, 1000, 8, 6, at, 0, none) == bad
