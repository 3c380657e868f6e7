"""What the sizes of the token attention's workspace say about how a call is laid out (no GPU)."""
import ctypes
import os

import pytest

from paper_2607_14898_amd import flashdecoder as fdb


def workspace(B, G, C, D, heads, n, dtype, weights=1, step=None):
    """Floats of workspace; dtype "f16", "bf16" or "f32"."""
    if not os.path.exists(fdb.LIB_PATH):
        pytest.skip("libflashdecoder.so not built")
    I3 = ctypes.c_int64 * 3
    step = step or D
    strides = I3(G * C * step, C * step, step)
    code = {"f32": fdb.FD_DTYPE_F32, "bf16": fdb.FD_DTYPE_BF16, "f16": fdb.FD_DTYPE_F16}[dtype]
    a = 1 << 20  # never read
    s = fdb.fd_token_cache(ctypes.sizeof(fdb.fd_token_cache), code, B, G, C, D, a, a, strides, strides, a, a)
    size = ctypes.c_size_t()
    st = fdb.load_library().fd_token_attend_workspace(ctypes.byref(s), heads, n, weights, ctypes.byref(size))
    assert st == fdb.FD_OK
    return size.value // 4


def up64(x):
    return (x + 63) // 64 * 64


def parts_floats(BG, parts, R, D):
    return up64(BG * parts * R * D) + up64(BG * parts * R * 2)


@pytest.mark.parametrize("C", [2 ** 18, 2 ** 22, 2 ** 24])
def test_single_tokens_part_long_caches(C):
    """Sums of a part of few rows end after 16384 slots."""
    got = workspace(1, 64, C, 32, 64, 1, "bf16", weights=0)
    parts = got / (64 * 34)
    assert parts >= C / 16384


@pytest.mark.parametrize("dtype,D,C", [("bf16", 32, 16385), ("f16", 128, 16385), ("f32", 64, 4097)])
def test_chunks_fold_long_caches(dtype, D, C):
    """Chunks without parts keep totals of their rows from 16384 (fp32: 4096) slots on, and nothing below."""
    heads, n = 32, 32768  # 8 x 1024 tiles of rows
    assert workspace(1, 8, C - 1, D, heads, n, dtype, weights=0) == 0
    assert workspace(1, 8, C, D, heads, n, dtype, weights=0) >= parts_floats(8, 1, 4 * n, D)


def test_many_rows_part_their_weights():
    """Sums of a weight end after 32768 rows."""
    heads, n, C = 4, 2 ** 18, 2 ** 18
    R = heads * n
    got = workspace(1, 1, C, 32, heads, n, "bf16") - workspace(1, 1, C, 32, heads, n, "bf16", weights=0)
    assert got >= up64(R) + up64(R // 32768 * C)


@pytest.mark.parametrize("dtype,D,held", [("f32", 64, 512), ("bf16", 64, 768), ("f16", 128, 512), ("f32", 128, 256)])
def test_single_tokens_fill_whole_rounds(dtype, D, held):
    """Parts of few rows make whole rounds of the workgroups that fit on 256 CUs at once."""
    G, C = 8, 65536
    got = workspace(1, G, C, D, 4 * G, 1, dtype, weights=0)
    fits = [s for s in range(1, 257) if parts_floats(G, s, 4, D) == got]
    assert len(fits) == 1 and fits[0] * G % held == 0


@pytest.mark.parametrize("B,G,C,n,chunks", [(1, 8, 131072, 1, 8), (1, 1, 1 << 24, 1, 1024), (4, 8, 262144, 1, 16),
                                            (1, 1, 100000, 1, 0), (8, 8, 131072, 1, 0), (16, 8, 262144, 1, 0),
                                            (1, 1, 131072, 0, 0)])
def test_one_token_among_many_slots(B, G, C, n, chunks):
    """Chunks of 16384 slots, four bytes each, where one workgroup a pair would leave the chip idle for long."""
    if not os.path.exists(fdb.LIB_PATH):
        pytest.skip("libflashdecoder.so not built")
    size = ctypes.c_size_t()
    assert fdb.load_library().fd_token_slots_workspace(B, G, C, n, ctypes.byref(size)) == fdb.FD_OK
    assert size.value == 4 * B * G * chunks
