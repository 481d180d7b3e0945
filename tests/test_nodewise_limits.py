"""Sizes beyond what a launch can have are refused before anything is written or sent to a device (host code only)."""
import ctypes

import pytest
import torch

from paper_2111_06483_amd import sar


@pytest.fixture(scope="module", autouse=True)
def built():
    sar.native()


def test_more_workgroups_than_a_launch_has():
    """Launches of 2^32 threads and more: layer norm of 64 rows a workgroup, packing of 128."""
    lib, none = sar.lib(), None
    err = lambda: lib.sar_last_error().decode()
    some = ctypes.create_string_buffer(512)
    at = (ctypes.addressof(some) + 255) // 256 * 256                # (never read: the calls are refused first)
    for dtype, rows in ((0, 64), (1, 128)):
        assert lib.sar_layernorm_fwd(at, none, none, 1e-5, at, none, dtype, rows << 24, 1, none, none, none, none, none) == sar.SAR_ERR_UNSUPPORTED
        assert "too many for one launch" in err()
    for dtype in (0, 1):
        assert lib.sar_pack(at, dtype, 1 << 32, 1, at, at, none) == sar.SAR_ERR_UNSUPPORTED and "too many" in err()
        assert lib.sar_unpack(at, at, dtype, 1 << 32, 1, at, none) == sar.SAR_ERR_UNSUPPORTED and "too many" in err()


def test_more_weights_than_a_launch_lays_out():
    """Refused where the scratch is asked for, and before a backward pass writes dW."""
    lib, none = sar.lib(), None
    n = ctypes.c_size_t()
    some = ctypes.create_string_buffer(512)
    at = (ctypes.addressof(some) + 255) // 256 * 256
    for K, F in ((1, 65536), (65536, 1)):
        assert lib.sar_linear_typed_workspace_bytes(1, K, F, 16384, ctypes.byref(n)) == sar.SAR_ERR_UNSUPPORTED
        assert "too many for one launch" in lib.sar_last_error().decode()
        assert lib.sar_linear_typed_workspace_bytes(1, K, F, 1024, ctypes.byref(n)) == 0
        assert lib.sar_linear_typed_bwd(at, none, none, at, at, at, 16384, 0, at + 16, at + 32, 0, 1, K, F, at, 1 << 62, none) == sar.SAR_ERR_UNSUPPORTED


def test_sizes_beyond_an_int():
    """A width of 2^32 + 8 is not one of 8.  (Tensors without rows or values: they take no memory.)"""
    wide = (1 << 32) + 8
    rows = lambda n, K: torch.empty(n, K)
    w, ptr = torch.empty(64, dtype=torch.uint8), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: sar.sar_pack(rows(0, wide), sar.packed_empty(0, wide, "cpu")),
                 lambda: sar.sar_unpack(sar.packed_empty(0, wide, "cpu"), rows(0, wide)),
                 lambda: sar.sar_layernorm_fwd(rows(0, wide), None, None, 1e-5, rows(0, wide)),
                 lambda: sar.sar_layernorm_bwd(rows(0, wide), rows(0, wide), rows(0, 2), None, False, rows(0, wide), None, None, None),
                 lambda: sar.sar_linear_typed_fwd(rows(0, wide), torch.empty(2, wide, 0), ptr, rows(0, 0), w),
                 lambda: sar.sar_linear_typed_fwd(rows(0, 0), torch.empty(2, 0, wide), ptr, rows(0, wide), w),
                 lambda: sar.sar_linear_typed_fwd(rows(0, 0), torch.empty(wide, 0, 4), ptr, rows(0, 4), w),
                 lambda: sar.sar_linear_typed_bwd(None, rows(0, 0), torch.empty(2, wide, 0), ptr, False, None, rows(0, wide), w),
                 lambda: sar.sar_linear_bwd_packed(None, rows(0, 0), torch.empty(wide, 0), False, None, rows(0, wide), w)):
        with pytest.raises(sar.SarError) as e:
            call()
        assert e.value.code == sar.SAR_ERR_UNSUPPORTED and str(wide) in str(e.value)
