"""Plain computations in 64 bits of the products in 8 bits and by group, and what rounding can make of them.

Tolerances.  HALF is half a step of an fp32 number, relative to it.  A product in 8 bits: the integer sum is exact, becomes a
float, and is multiplied by two scales: three roundings; where a launch splits K in halves both have three and their addition is one
more.  So |error| <= 4 HALF sa sb sum |a||b|.  The fused call's additions of the incoming partial (two, if split)
round numbers up to |incoming| + |result|.  A product of bf16: the products are exact in fp32, the K additions each round a
partial sum of at most sum |a||b|.  (1.001: products of roundings.)"""
import numpy as np
import torch

HALF = 2.0 ** -24
MORE = 1.001


def rows8(x):
    """t3_quant_rows of x (float64): integers, scales as fp32."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x).max(axis=1, initial=0.0)
    bad = ~np.isfinite(x).all(axis=1)
    q = np.rint(np.where(bad[:, None], 0.0, x) * 127.0 / np.where((a > 0) & ~bad, a, 1.0)[:, None])
    scale = (np.where(bad, np.nan, a).astype(np.float32) / np.float32(127.0)).astype(np.float32)
    return q.astype(np.int8), scale


def product8(a, sa, b, sb):
    """C and its bound, float64, of int8 tensors on the GPU."""
    a, b = a.double(), b.double()
    unit = torch.outer(sa.double(), sb.double())
    return a @ b.t() * unit, 4 * HALF * MORE * (a.abs() @ b.abs().t()) * unit.abs()


def spans(offsets, rows):
    """Rows of every group as the kernels read the offsets: never outside the rows, never back."""
    at, out = min(max(int(offsets[0]), 0), rows), []
    for end in offsets[1:]:
        end = max(min(max(int(end), 0), rows), at)
        out.append((at, end))
        at = end
    return out


def close(got, want, bound):
    """Whether got is within bound of want; NaN where want is."""
    got, nan = got.double(), want.isnan()
    assert torch.equal(got.isnan(), nan)
    far = ((got - want).abs() - bound).masked_fill(nan, -1.0)
    assert far.numel() == 0 or float(far.max()) <= 0.0, (float(far.max()), int((far > 0).sum()), [int(i) for i in (far > 0).nonzero()[0]])


_choice = None


def grouped_tile(wgrad, kn, M, N, K, groups, cus=256, wide_ok=True):
    """(wide-tile kernel, tile rows, tile columns, a last round may be cut in quarters) of a product by group, K in 2-byte elements."""
    global _choice
    if _choice is None:
        import ctypes
        import os
        import subprocess
        import tempfile
        here = os.path.dirname(os.path.abspath(__file__))
        root = os.path.dirname(here)
        with tempfile.TemporaryDirectory() as d:
            so = os.path.join(d, "grouped_choice.so")
            subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(root, "include"), "-I",
                            os.path.join(root, "paper_2401_16677_amd", "csrc"), os.path.join(here, "grouped_choice.cpp"), "-o", so], check=True)
            _choice = ctypes.CDLL(so)
        _choice.grouped_tile.argtypes = [ctypes.c_int] * 2 + [ctypes.c_int64] * 4 + [ctypes.c_int] * 2 + [ctypes.c_void_p]
    import ctypes
    out = (ctypes.c_int32 * 4)()
    _choice.grouped_tile(int(wgrad), int(kn), M, N, K, groups, cus, int(wide_ok), ctypes.cast(out, ctypes.c_void_p))
    return bool(out[0]), out[1], out[2], bool(out[3])


def quarters(counts, N, tile, places=256):
    """(tiles of the groups, those of the last round that are done in quarters)"""
    T = sum(-(-n // tile[0]) for n in counts) * -(-N // tile[1])
    return T, T % places if T > places and 2 * (T % places) <= places else 0


def grouped_wide_fits(kn, K, lda, ldb, ldc):
    """Whether the wide-tile kernel's offsets reach all of a forward product by group."""
    import ctypes
    grouped_tile(False, kn, 1, 8, 8, 1)               # (built)
    _choice.grouped_wide_fits.argtypes = [ctypes.c_int] + [ctypes.c_int64] * 4
    return bool(_choice.grouped_wide_fits(int(kn), K, lda, ldb, ldc))
