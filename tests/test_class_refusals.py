"""What the calls around a network's logits refuse, before anything reaches a device (tensors in host memory serve for that), and their scratch."""
import ctypes

import pytest
import torch

from paper_2111_06483_amd import sar

F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32
BAD, UNSUPPORTED = sar.SAR_ERR_INVALID_ARG, sar.SAR_ERR_UNSUPPORTED


@pytest.fixture(scope="module", autouse=True)
def built():
    sar.native()


def t(*shape, dtype=F32):
    return torch.zeros(*shape, dtype=dtype)


def refused(call, text, code=BAD):
    with pytest.raises(sar.SarError) as e:
        call()
    assert e.value.code == code and text in str(e.value), str(e.value)


def of(call, **defaults):
    return lambda **k: call(*{**defaults, **k}.values())


def calls():
    top = (t(4, 3), t(4, 3, dtype=I32))
    w = t(1 << 20, dtype=torch.uint8)
    return {
        "act_fwd": of(sar.sar_linear_act_fwd, X=t(4, 8), W=t(8, 6), bias=t(6), res=t(4, 6), act=1, after=False, Y=t(4, 6), A=t(4, 6), work=w),
        "act_bwd": of(sar.sar_linear_act_bwd, dY=t(4, 6), A=t(4, 6), X=t(4, 8), W=t(8, 6), act=1, acc=False, dW=t(8, 6), db=t(6), dX=t(4, 8), dA=t(4, 6), work=w),
        "logp_fwd": of(sar.sar_logprob_fwd, X=t(4, 8), label=t(4, dtype=I32), logp=t(4), lse=t(4), entropy=t(4), top=top, work=None),
        "logp_bwd": of(sar.sar_logprob_bwd, X=t(4, 8), label=t(4, dtype=I32), lse=t(4), entropy=t(4), dlogp=t(4), dentropy=t(4), dX=t(4, 8)),
        "distill_fwd": of(sar.sar_distill_fwd, X=t(4, 8), top=top, T=1.0, loss=t(4), lse=t(4), work=None),
        "distill_bwd": of(sar.sar_distill_bwd, X=t(4, 8), top=top, T=1.0, lse=t(4), dloss=t(4), dX=t(4, 8)),
    }


def test_tensors_in_host_memory():
    for call in calls().values():
        refused(call, "host memory")


def test_shapes_that_do_not_fit():
    c = calls()
    for name, wrong in (("W", t(7, 6)), ("bias", t(5)), ("res", t(4, 5)), ("Y", t(3, 6)), ("A", t(4, 7))):
        refused(lambda: c["act_fwd"](**{name: wrong}), name + " has shape")
    for name, wrong in (("A", t(4, 5)), ("X", t(3, 8)), ("W", t(8, 5)), ("dW", t(6, 8)), ("db", t(8)), ("dX", t(4, 6)), ("dA", t(5, 6))):
        refused(lambda: c["act_bwd"](**{name: wrong}), name + " has shape")
    for name, wrong in (("label", t(5, dtype=I32)), ("logp", t(4, 1)), ("lse", t(3)), ("entropy", t(8))):
        refused(lambda: c["logp_fwd"](**{name: wrong}), name + " has shape")
    for name, wrong in (("label", t(3, dtype=I32)), ("lse", t(5)), ("entropy", t(5)), ("dlogp", t(1)), ("dentropy", t(1)), ("dX", t(4, 7))):
        refused(lambda: c["logp_bwd"](**{name: wrong}), name + " has shape")
    for name, wrong in (("loss", t(5)), ("lse", t(4, 4))):
        refused(lambda: c["distill_fwd"](**{name: wrong}), name + " has shape")
    for name, wrong in (("lse", t(5)), ("dloss", t(5)), ("dX", t(8, 4))):
        refused(lambda: c["distill_bwd"](**{name: wrong}), name + " has shape")
    for name in ("logp_fwd", "distill_fwd", "distill_bwd"):
        refused(lambda: c[name](top=(t(5, 3), t(4, 3, dtype=I32))), "top values has shape")
        refused(lambda: c[name](top=(t(4, 3), t(4, 2, dtype=I32))), "top classes has shape")
        refused(lambda: c[name](top=t(4, 3)), "a pair (values, classes)")
        refused(lambda: c[name](top=(t(4, 3),)), "a pair (values, classes)")
    for name in ("distill_fwd", "distill_bwd"):
        refused(lambda: c[name](top=None), "a pair (values, classes)")


def test_types_that_do_not_fit():
    c = calls()
    refused(lambda: c["act_fwd"](X=t(4, 8, dtype=torch.float16)), "torch.float16", UNSUPPORTED)
    refused(lambda: c["act_fwd"](W=t(8, 6, dtype=BF16)), "W is torch.bfloat16")
    refused(lambda: c["act_fwd"](res=t(4, 6, dtype=BF16)), "res is torch.bfloat16")
    refused(lambda: c["act_bwd"](A=t(4, 6, dtype=BF16)), "A is torch.bfloat16")
    refused(lambda: c["act_bwd"](db=t(6, dtype=BF16)), "db is torch.bfloat16")
    refused(lambda: c["logp_fwd"](X=t(4, 8, dtype=torch.float64)), "torch.float64", UNSUPPORTED)
    refused(lambda: c["logp_fwd"](label=t(4, dtype=torch.int64)), "label is torch.int64")
    refused(lambda: c["logp_fwd"](top=(t(4, 3), t(4, 3, dtype=torch.int64))), "top classes is torch.int64")
    refused(lambda: c["logp_bwd"](dX=t(4, 8, dtype=BF16)), "dX is torch.bfloat16")
    refused(lambda: c["distill_bwd"](top=(t(4, 3, dtype=BF16), t(4, 3, dtype=I32))), "top values is torch.bfloat16")
    with pytest.raises(ValueError):
        c["logp_fwd"](X=t(8))
    with pytest.raises(ValueError):
        c["act_fwd"](W=t(2, 8, 6))
    with pytest.raises(AttributeError):
        c["distill_bwd"](lse=None)
    with pytest.raises(AttributeError):
        c["logp_bwd"](dX=None)


def test_tensors_that_are_no_plain_memory():
    c = calls()
    refused(lambda: c["act_fwd"](X=t(8, 4).T), "X must be contiguous")
    refused(lambda: c["act_bwd"](dA=t(4, 12)[:, ::2]), "dA must be contiguous")
    refused(lambda: c["logp_fwd"](logp=t(8)[::2]), "logp must be contiguous")
    refused(lambda: c["logp_fwd"](top=(t(3, 4).T, t(4, 3, dtype=I32))), "top values must be contiguous")
    refused(lambda: c["distill_bwd"](dX=t(4, 16)[:, 8:]), "dX must be contiguous")


def test_sizes_beyond_an_int():
    wide = (1 << 32) + 8
    rows = lambda n, C: torch.empty(n, C)
    none = (rows(0, 2), torch.empty(0, 2, dtype=I32))
    w = t(64, dtype=torch.uint8)
    for call in (lambda: sar.sar_linear_act_fwd(rows(0, wide), torch.empty(wide, 0), None, None, 0, False, rows(0, 0), None, w),
                 lambda: sar.sar_linear_act_bwd(rows(0, wide), None, None, torch.empty(0, wide), 0, False, None, None, rows(0, 0), None, w),
                 lambda: sar.sar_logprob_fwd(rows(0, wide), None, None, None, None),
                 lambda: sar.sar_logprob_bwd(rows(0, wide), None, rows(0, 1).view(0), None, None, None, rows(0, wide)),
                 lambda: sar.sar_distill_fwd(rows(0, wide), none, 1.0, None, None),
                 lambda: sar.sar_distill_bwd(rows(0, wide), none, 1.0, torch.empty(0), torch.empty(0), rows(0, wide))):
        refused(call, str(wide), UNSUPPORTED)
    refused(lambda: sar.sar_linear_act_fwd(rows(0, 8), torch.empty(8, 6), None, None, 1 << 33, False, rows(0, 6), None, w), str(1 << 33), UNSUPPORTED)


@pytest.fixture(scope="module")
def at():
    some = ctypes.create_string_buffer(1 << 16)
    yield (ctypes.addressof(some) + 255) // 256 * 256                # (never read: the calls are refused first)


def says(text):
    return text in sar.lib().sar_last_error().decode()


def test_errors_of_the_transform(at):
    lib, none, much = sar.lib(), None, 1 << 40
    fwd = lambda X=at, W=at + 4096, bias=none, res=none, act=1, after=0, Y=at + 8192, A=none, dtype=0, n=4, K=8, F=6, work=at, wb=much: \
        lib.sar_linear_act_fwd(X, W, bias, res, act, after, Y, A, dtype, n, K, F, work, wb, none)
    assert fwd(act=5) == UNSUPPORTED and says("SAR_ACT") and fwd(act=-1) == UNSUPPORTED
    assert fwd(dtype=2) == UNSUPPORTED and fwd(n=-1) == BAD and fwd(K=0) == BAD and fwd(F=0) == BAD
    assert fwd(K=65537) == UNSUPPORTED and fwd(F=65537) == UNSUPPORTED and fwd(n=(1 << 31) - 256) == UNSUPPORTED
    assert fwd(work=none) == BAD and says("needs") and fwd(wb=16) == BAD and fwd(work=at + 4) == BAD and says("16-byte")
    for k in ("X", "W", "Y"):
        assert fwd(**{k: none}) == BAD and says("null")
    assert fwd(Y=at) == BAD and says("alias") and fwd(Y=at + 4) == BAD and fwd(A=at + 8192) == BAD and fwd(A=at + 4096) == BAD
    assert fwd(res=at + 8196) == BAD and says("overlaps")
    assert fwd(res=at + 12288, A=at + 12288, after=1) == BAD and says("overlaps")
    assert fwd(n=0, X=none, W=none, Y=none) == 0
    bwd = lambda dY=at, A=at + 800, X=at + 1600, W=at + 2400, act=1, acc=0, dW=at + 3200, db=at + 4000, dX=at + 4800, dA=at + 5600, dtype=0, n=4, K=8, F=6, work=at, \
        wb=much: lib.sar_linear_act_bwd(dY, A, X, W, act, acc, dW, db, dX, dA, dtype, n, K, F, work, wb, none)
    assert bwd(act=7) == UNSUPPORTED and bwd(dtype=3) == UNSUPPORTED and bwd(work=none) == BAD and bwd(wb=8) == BAD
    assert bwd(dY=none) == BAD and bwd(A=none) == BAD and bwd(X=none) == BAD and bwd(W=none) == BAD and says("null")
    for other in (at, at + 800, at + 1600, at + 2400, at + 5600):
        assert bwd(dX=other) == BAD and says("dX must not alias")
    for other in (at, at + 800, at + 1600):
        assert bwd(dA=other) == BAD and says("dA must not alias")
    assert bwd(dW=at + 2400) == BAD and says("dW must not alias")
    size = ctypes.c_size_t()
    assert lib.sar_linear_act_workspace_bytes(4, 8, 6, none) == BAD and lib.sar_linear_act_workspace_bytes(-1, 8, 6, ctypes.byref(size)) == BAD
    # the calls that there were before take their own activations alone
    assert lib.sar_act_bwd(at, at, 2, at, 0, 8, none) == UNSUPPORTED and lib.sar_spmm_end(none, 0, none, none, 3, none, 0, 4, 8, none) == UNSUPPORTED


def test_errors_of_rows_of_scores(at):
    lib, none, size = sar.lib(), None, ctypes.c_size_t()
    fwd = lambda X=at, label=at, logp=at, lse=at, H=at, k=2, v=at, i=at, dtype=0, n=4, C=8, work=none, wb=0: \
        lib.sar_logprob_fwd(X, label, logp, lse, H, k, v, i, dtype, n, C, work, wb, none)
    assert fwd(dtype=2) == UNSUPPORTED and fwd(n=-1) == BAD and fwd(C=0) == BAD and fwd(k=-1) == BAD
    assert fwd(k=65) == UNSUPPORTED and says("at most 64") and fwd(C=(1 << 30) + 1) == UNSUPPORTED
    assert fwd(X=none) == BAD and fwd(label=none) == BAD and fwd(v=none) == BAD and fwd(i=none) == BAD and says("null")
    assert fwd(n=0, X=none, label=none, logp=none, v=none, i=none) == 0
    assert fwd(C=65536) == BAD and says("needs") and fwd(C=65536, work=at + 4, wb=1 << 30) == BAD and says("16-byte")
    bwd = lambda X=at, label=at, lse=at, H=at, dl=at, dh=at, dX=at, dtype=0, n=4, C=8: lib.sar_logprob_bwd(X, label, lse, H, dl, dh, dX, dtype, n, C, none)
    assert bwd(dtype=2) == UNSUPPORTED and bwd(n=-1) == BAD and bwd(C=0) == BAD
    for k in ("X", "lse", "dX", "label", "H"):
        assert bwd(**{k: none}) == BAD and says("null")
    assert bwd(n=0, X=none, lse=none, dX=none) == 0
    dfwd = lambda X=at, k=2, v=at, i=at, T=1.0, loss=at, lse=at, dtype=0, n=4, C=8, work=none, wb=0: \
        lib.sar_distill_fwd(X, k, v, i, T, loss, lse, dtype, n, C, work, wb, none)
    dbwd = lambda X=at, k=2, v=at, i=at, T=1.0, lse=at, dl=at, dX=at, dtype=0, n=4, C=8: lib.sar_distill_bwd(X, k, v, i, T, lse, dl, dX, dtype, n, C, none)
    for call in (dfwd, dbwd):
        for T in (0.0, -1.0, float("inf"), float("nan"), 1e-40):
            assert call(T=T) == BAD and says("temperature")
        assert call(dtype=2) == UNSUPPORTED and call(k=65) == UNSUPPORTED and call(k=-1) == BAD and call(C=0) == BAD
        assert call(X=none) == BAD and call(v=none) == BAD and call(i=none) == BAD and says("null")
        assert call(n=0, X=none) == 0
    assert dbwd(lse=none) == BAD and dbwd(dl=none) == BAD and dbwd(dX=none) == BAD
    assert dfwd(C=65536) == BAD and says("needs")
    for f in (lib.sar_logprob_workspace_bytes, lib.sar_distill_workspace_bytes):
        assert f(4, 8, 2, none) == BAD and f(-1, 8, 2, ctypes.byref(size)) == BAD and f(4, 8, 65, ctypes.byref(size)) == UNSUPPORTED
        assert f(4, 8, 2, ctypes.byref(size)) == 0 and size.value == 0


def counts():
    some = {n + d for k in range(5, 21) for n in (1 << k, 3 << (k - 1)) for d in (-1, 0, 1, 31, 32, 33)}
    return sorted(some | set(range(0, 1100)))


@pytest.mark.parametrize("C,k", [(47, 8), (2049, 1), (5000, 64), (8193, 0), (65_536, 8), (1 << 30, 64)])
def test_scratch_of_more_rows_serves_fewer(C, k):
    for f in (sar.sar_logprob_workspace_bytes, sar.sar_distill_workspace_bytes):
        sizes = [f(n, C, k) for n in counts()]
        assert sizes == sorted(sizes)


@pytest.mark.parametrize("K,F", [(1, 1), (47, 200), (100, 47), (128, 128), (100, 256), (256, 256), (512, 512), (1024, 96), (65_536, 1)])
def test_scratch_of_the_transform_grows_with_the_rows(K, F):
    sizes = [sar.sar_linear_act_workspace_bytes(n, K, F) for n in counts()]
    assert sizes == sorted(sizes)


def test_the_gradient_in_the_place_of_the_weights(at):
    lib = sar.lib()
    bwd = lambda dA, W=at + 2400, dX=at + 4800: lib.sar_linear_act_bwd(at, at + 800, at + 1600, W, 1, 0, at + 3200, at + 4000, dX, dA, 0, 4, 8, 6, at, 1 << 40, None)
    # (W: 192 bytes, dA: 96)
    for dA in (at + 2400, at + 2308, at + 2588):
        assert bwd(dA) == BAD and says("dA must not alias")


@pytest.mark.parametrize("T", [3.0e-39, 3.5e-39, 4.2e-39])
def test_temperatures_whose_exponents_have_no_factor(at, T):
    """1 / T is a number of 32 bits, log2(e) / T is none."""
    lib, none = sar.lib(), None
    assert lib.sar_distill_fwd(at, 2, at, at, T, at, at, 0, 4, 8, none, 0, none) == BAD and says("temperature")
    assert lib.sar_distill_bwd(at, 2, at, at, T, at, at, at, 0, 4, 8, none) == BAD and says("temperature")


@pytest.mark.parametrize("dtype,size", [(0, 4), (1, 2)])
def test_gradients_that_lie_across_the_scores(at, dtype, size):
    """In the scores' place or beside them, not shifted: other rows' scores would be read after they are overwritten."""
    lib, none, n, C = sar.lib(), None, 4, 8
    X, far = at + 4096, at + 16384
    for by in (-n * C * size + size, -C * size, -size, size, C * size, n * C * size - size):
        assert lib.sar_logprob_bwd(X, far, far, far, far, far, X + by, dtype, n, C, none) == BAD and says("overlaps")
        assert lib.sar_distill_bwd(X, 2, far, far, 1.0, far, far, X + by, dtype, n, C, none) == BAD and says("overlaps")


@pytest.mark.parametrize("n,K,F", [(4, 8, 6), (1 << 20, 256, 256)])
def test_scratch_that_the_forward_pass_needs(at, n, K, F):
    lib, none = sar.lib(), None
    size = sar.sar_linear_typed_workspace_bytes(n, K, F, 1)
    assert lib.sar_linear_act_fwd(at, at, none, none, 1, 0, at, none, 0, n, K, F, at, size - 1, none) == BAD and says(f"needs {size}")
