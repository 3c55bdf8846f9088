"""Arguments of the products in 8 bits and by group that are refused before anything is launched; no GPU needed."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2401_16677_amd import binding as t3
from products import grouped_wide_fits, rows8, spans

FAKE = 0x10000


def status(call, *args):
    try:
        call(*args, stream=0)
    except t3.T3Error as e:
        return e.status
    return t3.T3_OK


def quant(rows=4, cols=64, x=FAKE, q=FAKE, s=FAKE, ldx=None, ldq=None, x_type=t3.T3_TYPE_BF16):
    return status(lambda **k: t3.t3_quant_rows(rows, cols, x, q, s, ldx=ldx, ldq=ldq, x_type=x_type, **k))


def test_rows_refused():
    assert quant(rows=0) == t3.T3_OK
    assert quant(x=None) == quant(q=None) == quant(s=None) == t3.T3_ERR_NULL
    assert quant(rows=-1) == quant(cols=-8) == quant(ldx=56) == quant(ldq=56) == quant(x_type=2) == t3.T3_ERR_BAD_SHAPE
    assert quant(cols=60, ldx=64, ldq=64) == quant(ldx=68) == quant(ldq=68) == quant(x=FAKE + 2) == quant(q=FAKE + 4) == quant(s=FAKE + 2) == t3.T3_ERR_ALIGN
    assert quant(ldx=66, x_type=t3.T3_TYPE_F32) == t3.T3_ERR_ALIGN
    assert quant(rows=1 << 30, ldx=1 << 61) == quant(rows=1 << 30, ldq=1 << 61) == t3.T3_ERR_UNSUPPORTED


GEMM = dict(M=256, N=1024, K=256, tp=4, rank=0, tile_m=128, tile_n=128)


def plain(A=FAKE, sa=FAKE, B=FAKE, sb=FAKE, C=FAKE, **kw):
    return status(t3.t3_gemm_i8, t3.problem(**{**GEMM, **kw}), A, sa, B, sb, C)


def fused(A=FAKE, sa=FAKE, B=FAKE, sb=FAKE, R=FAKE, fwd=FAKE, track=FAKE, **kw):
    return status(t3.t3_gemm_rs_fused_i8, t3.problem(**{**GEMM, **kw}), A, sa, B, sb, R, fwd, track)


@pytest.mark.parametrize("call", [plain, fused])
def test_products_in_8_bits_refused(call):
    assert call(M=0) == call(N=0) == t3.T3_OK
    assert call(A=None) == call(sa=None) == call(B=None) == call(sb=None) == t3.T3_ERR_NULL
    assert call(M=-1) == call(rank=4) == call(N=1022) == call(lda=240) == call(ldb=240) == call(a_layout=2) == call(b_layout=2) == t3.T3_ERR_BAD_SHAPE
    assert call(tile_m=96) == t3.T3_ERR_BAD_TILE
    assert call(K=248) == call(lda=264) == call(ldb=264) == call(A=FAKE + 8) == call(B=FAKE + 8) == call(sa=FAKE + 2) == call(sb=FAKE + 1) == t3.T3_ERR_ALIGN
    assert call(b_layout=t3.T3_B_KN, ldb=1024) == call(a_layout=t3.T3_A_KM, lda=256) == call(K=131072) == t3.T3_ERR_UNSUPPORTED
    assert call(tile_begin=1) == call(tile_limit=5) == t3.T3_ERR_UNSUPPORTED      # (16 tiles a ring step)
    assert call(M=1 << 20, K=4096) == t3.T3_ERR_UNSUPPORTED                        # A of 2^32 bytes
    assert call(lda=1 << 60) == call(ldb=1 << 60) == t3.T3_ERR_UNSUPPORTED         # (times M no 64-bit number)
    lib = t3.lib()
    assert lib.t3_gemm_i8(None, FAKE, FAKE, FAKE, FAKE, FAKE, 0) == t3.T3_ERR_NULL
    assert lib.t3_gemm_rs_fused_i8(None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 0) == t3.T3_ERR_NULL


def test_results_of_products_in_8_bits_refused():
    assert plain(C=None) == fused(R=None) == fused(fwd=None) == fused(track=None) == t3.T3_ERR_NULL
    assert plain(ldc=1000) == fused(ldr=1000) == t3.T3_ERR_BAD_SHAPE
    assert plain(ldc=1026) == plain(C=FAKE + 4) == fused(R=FAKE + 4) == fused(N=1016) == t3.T3_ERR_ALIGN
    assert fused(flags=t3.T3_FLAG_TWO_WRITERS) == fused(flags=16) == fused(split_k=2) == t3.T3_ERR_UNSUPPORTED


GROUPED = dict(rows=100, groups=4, N=64, K=128)


def grouped(o=FAKE, A=FAKE, B=FAKE, C=FAKE, **kw):
    return status(t3.t3_gemm_grouped, t3.grouped(**{**GROUPED, **kw}), o, A, B, C)


def grouped8(o=FAKE, A=FAKE, sa=FAKE, B=FAKE, sb=FAKE, C=FAKE, **kw):
    return status(t3.t3_gemm_grouped_i8, t3.grouped(**{**GROUPED, **kw}), o, A, sa, B, sb, C)


def wgrad(o=FAKE, A=FAKE, B=FAKE, C=FAKE, **kw):
    return status(t3.t3_gemm_grouped_wgrad, t3.grouped(**{**GROUPED, **kw}), o, A, C, B)


@pytest.mark.parametrize("call", [grouped, grouped8, wgrad])
def test_groups_refused(call):
    assert call(o=None) == call(A=None) == call(B=None) == call(C=None) == t3.T3_ERR_NULL
    assert call(rows=-1) == call(groups=0) == call(N=-4) == call(K=-8) == call(b_layout=2) == t3.T3_ERR_BAD_SHAPE
    assert call(lda=120) == call(ldb=120) == call(ldc=60) == call(stride_b=-8) == t3.T3_ERR_BAD_SHAPE
    assert call(groups=257) == call(flags=2) == t3.T3_ERR_UNSUPPORTED
    assert call(K=124) == call(N=62) == call(lda=130) == call(ldc=66) == call(ldb=130) == call(stride_b=64 * 128 + 2) == t3.T3_ERR_ALIGN
    assert call(o=FAKE + 2) == call(A=FAKE + 8) == call(B=FAKE + 8) == call(C=FAKE + 8) == t3.T3_ERR_ALIGN
    assert call(lda=1 << 60) == call(ldb=1 << 60) == call(ldc=1 << 60) == call(stride_b=1 << 60) == t3.T3_ERR_UNSUPPORTED
    assert call(rows=1 << 25, K=256) == call(rows=1 << 25, N=64, ldc=128) == t3.T3_ERR_UNSUPPORTED or call is grouped8
    assert call(N=0) == t3.T3_OK


def test_groups_refused_by_one_call():
    assert grouped(b_layout=t3.T3_B_KN, K=100) == grouped(b_layout=t3.T3_B_KN, N=60) == t3.T3_ERR_ALIGN
    assert grouped(flags=t3.T3_GROUPED_ACCUMULATE) == grouped8(flags=t3.T3_GROUPED_ACCUMULATE) == t3.T3_ERR_UNSUPPORTED
    assert grouped8(b_layout=t3.T3_B_KN) == grouped8(K=131072) == grouped8(rows=1 << 25, K=128) == t3.T3_ERR_UNSUPPORTED
    assert grouped8(sa=None) == grouped8(sb=None) == t3.T3_ERR_NULL
    assert grouped8(K=120) == grouped8(lda=136) == grouped8(sa=FAKE + 2) == grouped8(sb=FAKE + 2) == t3.T3_ERR_ALIGN
    assert wgrad(stride_b=64 * 128 - 4) == wgrad(stride_b=0) == t3.T3_ERR_BAD_SHAPE     # groups' results over one another
    assert wgrad(N=60, ldc=64) == wgrad(K=120, lda=124, ldb=128) == t3.T3_ERR_ALIGN
    assert grouped(rows=0) == grouped8(rows=0) == wgrad(K=0) == t3.T3_OK
    lib = t3.lib()
    assert lib.t3_gemm_grouped(None, FAKE, FAKE, FAKE, FAKE, 0) == t3.T3_ERR_NULL
    assert lib.t3_gemm_grouped_i8(None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 0) == t3.T3_ERR_NULL
    assert lib.t3_gemm_grouped_wgrad(None, FAKE, FAKE, FAKE, FAKE, 0) == t3.T3_ERR_NULL


def test_struct_layout():
    assert ctypes.sizeof(t3.T3Grouped) == 6 * 4 + 4 * 8 and t3.T3Grouped.lda.offset == 24 and t3.T3Grouped.stride_b.offset == 48


def test_the_tests_own_reading_of_rows_and_offsets():
    q, s = rows8(np.array([[127.0, 0.5, 1.5, -2.5], [0, 0, 0, 0], [np.nan, 1, 1, 1]]))
    assert q.tolist() == [[127, 0, 2, -2], [0] * 4, [0] * 4] and s[0] == 1.0 and s[1] == 0.0 and np.isnan(s[2])
    assert spans([5, 2, 30, 30], 40) == [(5, 5), (5, 30), (30, 30)]
    assert spans([-4, 10, 2000000000, 3], 25) == [(0, 10), (10, 25), (25, 25)]


def test_arrays_without_elements_need_no_address():
    """A rank that got no rows has tensors without elements, whose address is 0."""
    none = [torch.empty(s, dtype=d) for s, d in [((0, 64), torch.bfloat16), ((0, 64), torch.int8), ((0,), torch.float32), ((0, 64), torch.float32)]]
    x, q, s, c = none
    assert all(t.data_ptr() == 0 for t in none)
    for y, t in ((x, t3.T3_TYPE_BF16), (c, t3.T3_TYPE_F32)):
        assert quant(rows=0, x=y, q=q, s=s, x_type=t) == t3.T3_OK
    assert plain(M=0, A=q, sa=s, C=c) == fused(M=0, A=q, sa=s, R=c, fwd=c) == t3.T3_OK
    assert plain(N=0, B=q, sb=s, C=c) == fused(N=0, B=q, sb=s, R=c, fwd=c) == t3.T3_OK
    assert grouped(rows=0, A=x, C=c) == grouped8(rows=0, A=q, sa=s, C=c) == t3.T3_OK
    assert grouped(N=0, B=x, C=c) == grouped8(N=0, B=q, sb=s, C=c) == t3.T3_OK
    assert wgrad(N=0, B=c, C=x) == wgrad(K=0, A=x, B=c) == t3.T3_OK
    # what has elements, or is written without any rows, is asked for still
    assert quant(cols=0, x=None, q=None, s=None) == plain(K=0, A=None, B=None, C=None) == plain(K=0, A=None, B=None, sa=None) == t3.T3_ERR_NULL
    assert fused(M=0, track=None) == grouped(rows=0, o=None) == wgrad(N=0, o=None) == t3.T3_ERR_NULL
    assert grouped(K=0, A=None, B=None, C=None) == grouped8(K=0, A=None, B=None, sa=None) == wgrad(rows=0, A=None, C=None, B=None) == t3.T3_ERR_NULL


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int8, torch.int16, torch.int32])
def test_rows_of_other_types_are_refused(dtype):
    """(Read as bfloat16 they would give integers and scales of other numbers.)"""
    x = torch.zeros((4, 64), dtype=dtype)
    with pytest.raises(TypeError, match=str(dtype)):
        t3.t3_quant_rows(0, 64, x, FAKE, FAKE, stream=0)
    for ok in (torch.bfloat16, torch.float32):
        t3.t3_quant_rows(0, 64, x.to(ok), FAKE, FAKE, stream=0)
    t3.t3_quant_rows(0, 64, FAKE, FAKE, FAKE, stream=0)


@pytest.mark.parametrize("cols", [256, 128])
def test_lanes_behind_a_short_contraction_stay_past_the_buffer(cols):
    """B stored K x N: the byte offsets of a slab's 64 k-rows, as the wide-tile kernel's 32-bit numbers, where it may be used: k-rows from K on, and
    columns from the tile's last on, are past the buffer (an infinity there times A's zeros would be NaN)."""
    fits = 0
    for K in (8, 16, 24, 56, 64):
        for ldb in [1 << e for e in range(12, 29)] + [(1 << 24) + 8, (1 << 25) - 8, 3 << 23, 5 << 24]:
            if K * ldb >= 1 << 31 or not grouped_wide_fits(True, K, K, ldb, 512):
                continue
            fits += 1
            k, col = np.arange(64, dtype=np.uint64)[:, None], np.arange(0, 256, 8, dtype=np.uint64)[None, :]
            off = (k * np.uint64(ldb) + col) * np.uint64(2) & np.uint64(0xFFFFFFFF)
            if cols < 256:                         # (lanes outside get the top bit, the others lose it)
                off = np.where(col >= cols, off | np.uint64(1 << 31), off & np.uint64((1 << 31) - 1))
            inside = off < K * ldb * 2
            assert np.array_equal(inside, np.broadcast_to((k < K) & (col < cols), inside.shape)), (K, ldb)
    assert fits > 50 and grouped_wide_fits(True, 64, 64, 1 << 24, 512) and not grouped_wide_fits(True, 65, 72, 1 << 24, 512)


def test_limits_of_groups_are_ones_of_sizes():
    """What the header says of sizes, whatever tiles are picked; no further limit (without a GPU a launch that is not refused ends in T3_ERR_HIP)."""
    launched = (t3.T3_OK, t3.T3_ERR_HIP)
    far = dict(N=1 << 24, K=8, ldc=1 << 24)           # rows of dC of 2^25 bytes
    assert wgrad(rows=300, groups=64, **far) == t3.T3_ERR_UNSUPPORTED          # dC of 2^31 elements and more
    assert wgrad(rows=0, groups=64, N=8, K=1 << 24, lda=1 << 24) == t3.T3_ERR_UNSUPPORTED     # 2^24 tiles of 64 x 64, (rows + 256) lda 2^32
    if torch.cuda.is_available():
        return
    assert wgrad(rows=4, groups=63, **far) in launched                         # (2^24 less 2^18 of them)
    assert wgrad(rows=4, groups=64, **{**far, "N": (1 << 24) - 64}) in launched
    assert grouped(rows=255, groups=256, N=4194300, K=8, stride_b=0) in launched
    assert grouped(rows=1, groups=256, N=(1 << 28) - 8, K=8, ldb=8, stride_b=0) in launched
    assert grouped(rows=(1 << 28) - 8, groups=256, N=4, K=8) in launched
