"""Sizes beyond what a launch can have are refused before anything is written or sent to a device (host code only)."""
import ctypes

import pytest

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
