"""Workspace sizes of the linear layer's calls and what is refused without one
(no GPU: every call here is refused)."""
import ctypes
import os

import pytest

from paper_1911_08907_amd import aps as A
from paper_1911_08907_amd import build as B
from tests.test_abi import GOOD, no_gpu

BF16, F32, F16 = A.APS_DTYPE_BF16, A.APS_DTYPE_F32, A.APS_DTYPE_F16
FWD, ON = A.APS_LINEAR_FORWARD, A.APS_LINEAR_ON_CHUNKS
BARE = FWD | ON | A.APS_LINEAR_NO_CKPT


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(A.LIB_PATH):
        B.build()
    return A.lib()


@pytest.mark.parametrize("dt", [BF16, F16, F32])
def test_calls_without_a_checkpoint(lib, dt):
    w = lib.aps_linear_workspace_bytes
    for M, N, K in ((1, 4096, 1024), (8, 4096, 1024), (16, 128, 128)):
        assert w(BARE, M, N, K, dt) == 0
    for M, N, K in ((1, 16, 65536), (32, 64, 65536), (33, 64, 65536), (64, 1024, 4096)):
        assert w(BARE, M, N, K, dt) == w(FWD, M, N, K, dt) > 0
    for op in range(3):
        # whole and split contractions; anything, where the rows may start anywhere
        assert w(op | ON, 2048, 2048, 2048, dt) in (0, w(op, 2048, 2048, 2048, dt))
        assert w(op | ON, *((64, 64, 65536), (64, 65536, 64), (65536, 64, 64))[op], dt) > 0
        assert w(op | A.APS_LINEAR_NO_CKPT, 8, 4096, 1024, dt) == w(op, 8, 4096, 1024, dt)
    # no operations
    assert w(3 | ON, 8, 64, 65536, dt) == 0 and w(64, 8, 64, 65536, dt) == 0 and w(-1, 8, 64, 65536, dt) == 0


@pytest.mark.parametrize("op", range(3))
def test_operands_off_their_chunks(lib, op):
    """More bytes where a copy pays: at most both operands' and the sums'."""
    w, off = lib.aps_linear_workspace_bytes, A.APS_LINEAR_OFF_CHUNKS
    assert w(op | off, 4096, 4096, 4096, BF16) >= w(op, 4096, 4096, 4096, BF16) + 4096 * 4096
    for M, N, K in ((1, 1, 1), (1, 4096, 1024), (40, 256, 128), (333, 1000, 520), (2000, 1001, 64), (0, 8, 8), (8, 8, 0)):
        for dt in (BF16, F16, F32):
            base, more = w(op, M, N, K, dt), w(op | off, M, N, K, dt)
            assert base <= more <= base + (M * N + N * K + M * K) * 4 + 64 * max(1, M, N, K) + 1024 + base


@no_gpu
def test_a_missing_workspace(lib):
    """NULL with 0 bytes is refused where the call would use some, NULL with
    bytes and a workspace too short wherever one can be needed."""
    def call(M, N, K, codes=None, ws=None, wb=0):
        f = A.Format(4, 3).c()
        return lib.aps_linear(GOOD, K, GOOD, K, None, None, 0, GOOD, N, M, N, K, BF16, 0, f, codes, N, codes, ws, wb, None)

    assert call(1, 16, 65536) == A.APS_ERR_NULL
    assert call(1, 64, 65536, codes=GOOD) == A.APS_ERR_NULL and call(64, 64, 65536) == A.APS_ERR_NULL
    assert call(1, 4096, 1024, wb=1 << 30) == A.APS_ERR_NULL
    assert call(1, 4096, 1024, ws=GOOD, wb=16) == A.APS_ERR_SIZE
    assert call(1, 4096, 1024, ws=ctypes.c_void_p(4097), wb=1 << 30) == A.APS_ERR_ALIGN
