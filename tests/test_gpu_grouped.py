"""Products by group (t3_gemm_grouped, its 8-bit form and the gradient of the weights) on the GPU against 64 bits."""
import pytest
import torch

from paper_2401_16677_amd import binding as t3
from products import HALF, MORE, close, grouped_tile, grouped_wide_fits, product8, quarters, rows8, spans

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
OUTSIDE = 77.0


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def offsets_of(counts, first=0):
    o = [first]
    for n in counts:
        o.append(o[-1] + n)
    return o


def device(offsets):
    return torch.tensor(offsets, dtype=torch.int32).to(DEV)


def bf16(g, *shape):
    return torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)


def sum_bound(a, b):
    """Of a.double() @ b.double() summed in fp32: see products."""
    return a.shape[1] * HALF * MORE * (a.double().abs() @ b.double().abs())


# counts, rows before the first group, rows behind the last
GROUPS = [([1], 0, 0), ([5], 0, 2), ([3, 0, 4], 0, 0), ([0, 0, 7, 0], 2, 1), ([1, 1], 0, 0), ([33, 64, 1, 128, 65], 0, 9), ([300, 0, 511, 257], 5, 0),
          ([2] * 64, 0, 0), ([0, 3] * 50, 1, 4), ([1] * 256, 0, 3), ([0] * 255 + [90], 0, 0), ([1000, 20], 0, 0), ([0, 0], 3, 0),
          ([700, 900, 1, 450], 0, 30)]
SIZES = {"nk": [(4, 8), (36, 72), (132, 520), (520, 136), (1028, 1288)], "kn": [(8, 8), (40, 128), (264, 584), (1032, 328)]}


def check_forward(counts, first, behind, N, K, kn, integers=False, pads=(0, 0, 0), shared=False):
    g = gen(N + K + len(counts))
    rows, E = first + sum(counts) + behind, len(counts)
    o = offsets_of(counts, first)
    pa, pb, pc = pads
    A = bf16(g, rows, K + pa)
    B = bf16(g, 1 if shared else E, *((K, N + pb) if kn else (N, K + pb)))
    if integers:                                    # every partial sum is a whole number below 2^24: exact in any order
        A, B = (A * 2).round().clamp(-8, 8), (B * 2).round().clamp(-8, 8)
    A[:first] = float("nan")                        # rows of no group
    A[o[-1]:] = float("nan")
    C = torch.full((rows, N + pc), OUTSIDE, device=DEV)
    p = t3.grouped(rows, E, N, K, b_layout=t3.T3_B_KN if kn else t3.T3_B_NK, lda=K + pa, ldb=(N if kn else K) + pb, ldc=N + pc,
                   stride_b=0 if shared else None)
    t3.t3_gemm_grouped(p, device(o), A, B, C)
    torch.cuda.synchronize()
    for e, (a, b) in enumerate(spans(o, rows)):
        w = B[0 if shared else e]
        w = w[:, :N] if kn else w[:, :K].t()
        x = A[a:b, :K]
        want = x.double() @ w.double()
        if integers:
            assert torch.equal(C[a:b, :N].double(), want)
        else:
            close(C[a:b, :N], want, sum_bound(x, w))
    assert bool((C[:first] == OUTSIDE).all()) and bool((C[o[-1]:] == OUTSIDE).all()) and bool((C[:, N:] == OUTSIDE).all())


@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("case", range(len(GROUPS)))
def test_forward(case, layout):
    counts, first, behind = GROUPS[case]
    for i, (N, K) in enumerate(SIZES[layout]):
        if sum(counts) * N * K * len(counts) > 4e9:
            continue
        print(counts[:8], first, behind, N, K, flush=True)
        check_forward(counts, first, behind, N, K, layout == "kn", integers=i % 2 == 1)


@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("counts", [[3, 0, 40], [300, 129, 600]])
def test_forward_strides_and_one_operand_for_all(layout, counts):
    check_forward(counts, 1, 2, 264, 192, layout == "kn", pads=(24, 40, 12))
    check_forward(counts, 0, 0, 264, 192, layout == "kn", integers=True, shared=True)


@pytest.mark.parametrize("N,K,counts", [(4096, 4096, [700, 300, 0, 1500]), (2048, 6144, [2, 0, 1, 5, 1, 1]), (2560, 1024, [2000, 1900])])
def test_forward_large(N, K, counts):
    check_forward(counts, 0, 17, N, K, False)
    check_forward(counts, 0, 0, N, K, True, integers=True)


@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("K", [8, 56, 64, 72, 128, 136])
def test_forward_short_contraction(layout, K):
    """K of one slab and of little more, in launches of several rounds."""
    check_forward([700, 900, 1, 450, 0, 1300], 2, 3, 2560, K, layout == "kn", integers=K % 16 == 0)


# rows of every group, and how many tiles of the last round are done in quarters (0: a full round, or one more than half full)
ROUNDS = [([3000, 2000, 500, 500], 64), ([1400, 1400, 1600, 1600], 112), ([0, 2900, 1, 1600, 1000, 500], 112), ([1600, 1600, 1800, 1300], 0), ([4096, 4096], 0)]


@pytest.mark.parametrize("layout", ["nk", "kn", "8 bits"])
@pytest.mark.parametrize("counts,cut", ROUNDS)
@pytest.mark.parametrize("N", [6144, 6104])
def test_last_round_in_quarters(counts, cut, N, layout):
    K, rows, E, kn = 1024, sum(counts), len(counts), layout == "kn"
    choice = grouped_tile(False, kn, rows + 3, N, K, E)
    assert choice == (True, 256, 256, True) and quarters(counts, N, (256, 256))[1] == cut
    if layout == "8 bits":
        g, o = gen(cut + N), offsets_of(counts, 1)
        A = torch.randint(-128, 128, (rows + 3, 2 * K), generator=g, device=DEV, dtype=torch.int8)
        B = torch.randint(-128, 128, (E, N, 2 * K), generator=g, device=DEV, dtype=torch.int8)
        sa, sb = torch.exp(torch.randn(rows + 3, generator=g, device=DEV)), torch.exp(torch.randn((E, N), generator=g, device=DEV))
        C = torch.full((rows + 3, N), OUTSIDE, device=DEV)
        t3.t3_gemm_grouped_i8(t3.grouped(rows + 3, E, N, 2 * K), device(o), A, sa, B, sb, C)
        for e, (a, b) in enumerate(spans(o, rows + 3)):
            close(C[a:b], *product8(A[a:b], sa[a:b], B[e], sb[e]))
        assert bool((C[:1] == OUTSIDE).all()) and bool((C[o[-1]:] == OUTSIDE).all())
    else:
        check_forward(counts, 1, 2, N, K, kn, integers=N % 256 == 0)


@pytest.mark.parametrize("layout", ["nk", "kn"])
def test_forward_of_many_groups(layout):
    counts = [183, 265, 302, 304, 311, 351, 356, 359, 404, 489, 541, 674, 750, 793, 953, 1155]
    N, K, kn = (1280, 2560, True) if layout == "kn" else (5120, 1280, False)
    check_forward(counts, 0, 0, N, K, kn)
    check_forward(counts[::-1], 0, 0, N - 8, K, kn, integers=True)


@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("add", [False, True])
def test_wgrad_last_round_in_quarters(layout, add):
    counts = [183, 265, 0, 606, 311, 351, 356, 359, 404, 489, 541, 674, 750, 793, 953, 1155]
    for N, K in [(5120, 1280), (5112, 1272)]:
        M, n = (K, N) if layout == "kn" else (N, K)
        choice = grouped_tile(True, True, M, n, sum(counts), 16)
        T = 16 * -(-M // choice[1]) * -(-n // choice[2])
        assert choice[3] and 0 < T % 256 <= 128
        check_wgrad(counts, 0, 0, N, K, layout == "kn", add, N == 5120)


def test_no_contraction_and_no_rows():
    C = torch.full((6, 8), OUTSIDE, device=DEV)
    x = torch.zeros(512, dtype=torch.bfloat16, device=DEV)
    t3.t3_gemm_grouped(t3.grouped(6, 2, 8, 0), device([0, 2, 5]), x, x, C)
    assert bool((C[:5] == 0.0).all()) and bool((C[5] == OUTSIDE).all())
    t3.t3_gemm_grouped(t3.grouped(0, 2, 8, 8), device([0, 0, 0]), x, x, C)
    t3.t3_gemm_grouped(t3.grouped(6, 2, 8, 8), device([6, 6, 6]), x, x, C)
    torch.cuda.synchronize()
    assert bool((C[:5] == 0.0).all()) and bool((C[5] == OUTSIDE).all())


def test_groups_further_apart_than_32_bits_count():
    """The second group's operand (and gradient) starts past 2^31 elements and 2^32 bytes."""
    N, K, rows, counts, stride = 64, 128, 40, [25, 15], (1 << 32) + 4096
    g, o = gen(6), offsets_of([25, 15])
    raw = torch.empty(2 * (stride + N * K), dtype=torch.int8, device=DEV)
    A, d = bf16(g, rows, K), bf16(g, rows, N)
    w = [bf16(g, N, K) for _ in counts]
    B = raw.view(torch.bfloat16)
    for e in range(2):
        B[e * stride:e * stride + N * K] = w[e].view(-1)
    C = torch.zeros((rows, N), device=DEV)
    t3.t3_gemm_grouped(t3.grouped(rows, 2, N, K, stride_b=stride), device(o), A, B, C)
    for e, (a, b) in enumerate(spans(o, rows)):
        close(C[a:b], A[a:b].double() @ w[e].double().t(), sum_bound(A[a:b], w[e].t()))
    q = [torch.randint(-128, 128, (N, K), generator=g, device=DEV, dtype=torch.int8) for _ in counts]
    x = torch.randint(-128, 128, (rows, K), generator=g, device=DEV, dtype=torch.int8)
    sa, sb = torch.ones(rows, device=DEV), torch.ones((2, N), device=DEV)
    for e in range(2):
        raw[e * stride:e * stride + N * K] = q[e].view(-1)
    t3.t3_gemm_grouped_i8(t3.grouped(rows, 2, N, K, stride_b=stride), device(o), x, sa, raw, sb, C)
    for e, (a, b) in enumerate(spans(o, rows)):
        close(C[a:b], *product8(x[a:b], sa[a:b], q[e], sb[e]))
    dB, apart = raw.view(torch.float32), (1 << 30) + 1024
    t3.t3_gemm_grouped_wgrad(t3.grouped(rows, 2, N, K, stride_b=apart), device(o), A, d, dB)
    for e, (a, b) in enumerate(spans(o, rows)):
        close(dB[e * apart:e * apart + N * K].view(N, K), d[a:b].double().t() @ A[a:b].double(), sum_bound(d[a:b].t(), A[a:b]))


BAD = [[5, 2, 30, 30], [-4, 10, 10, 25], [0, 10, 2000000000, 3], [-2147483648, 2147483647, 0, 40], [40, 30, 20, 10], [3, 0, 0, 0]]


@pytest.mark.parametrize("o", BAD)
def test_offsets_out_of_order_or_range_are_read_as_the_nearest(o):
    """(Results by the offsets as the header says they are read; products.spans is checked without a GPU.)"""
    rows, E, N, K = 40, 3, 64, 64
    g = gen(2)
    A, B, dC = bf16(g, rows, K), bf16(g, E, N, K), bf16(g, rows, N)
    C, dB = torch.full((rows, N), OUTSIDE, device=DEV), torch.full((E, N, K), OUTSIDE, device=DEV)
    t3.t3_gemm_grouped(t3.grouped(rows, E, N, K), device(o), A, B, C)
    t3.t3_gemm_grouped_wgrad(t3.grouped(rows, E, N, K), device(o), A, dC, dB)
    torch.cuda.synchronize()
    left = torch.ones(rows, dtype=torch.bool, device=DEV)
    for e, (a, b) in enumerate(spans(o, rows)):
        close(C[a:b], A[a:b].double() @ B[e].double().t(), sum_bound(A[a:b], B[e].t()))
        close(dB[e], dC[a:b].double().t() @ A[a:b].double(), sum_bound(dC[a:b].t(), A[a:b]))
        left[a:b] = False
    assert bool((C[left] == OUTSIDE).all())


# ------------------------------------------------------------------ 8 bits

@pytest.mark.parametrize("case", range(len(GROUPS)))
def test_in_8_bits(case):
    counts, first, behind = GROUPS[case]
    rows, E = first + sum(counts) + behind, len(counts)
    for N, K, pad in [(4, 16, 0), (36, 80, 16), (132, 528, 0), (1028, 1296, 32)]:
        if sum(counts) * N * K * E > 4e9:
            continue
        g = gen(case * 7 + K)
        A = torch.randint(-128, 128, (rows, K + pad), generator=g, device=DEV, dtype=torch.int8)
        B = torch.randint(-128, 128, (E, N, K + pad), generator=g, device=DEV, dtype=torch.int8)
        sa, sb = torch.exp(torch.randn(rows, generator=g, device=DEV)), torch.exp(torch.randn((E, N), generator=g, device=DEV))
        o = offsets_of(counts, first)
        sa[:first], sa[o[-1]:] = float("nan"), float("nan")
        C = torch.full((rows, N + 4), OUTSIDE, device=DEV)
        t3.t3_gemm_grouped_i8(t3.grouped(rows, E, N, K, lda=K + pad, ldb=K + pad, ldc=N + 4), device(o), A, sa, B, sb, C)
        torch.cuda.synchronize()
        for e, (a, b) in enumerate(spans(o, rows)):
            close(C[a:b, :N], *product8(A[a:b, :K], sa[a:b], B[e][:, :K], sb[e]))
        assert bool((C[:first] == OUTSIDE).all()) and bool((C[o[-1]:] == OUTSIDE).all()) and bool((C[:, N:] == OUTSIDE).all())


@pytest.mark.parametrize("N,K,counts", [(4096, 2048, [700, 300, 0, 1500]), (2048, 6144, [2, 0, 1, 5, 1, 1]), (2560, 1024, [2000, 1900]),
                                        (2560, 112, [900, 1, 0, 2500]), (2560, 128, [900, 1, 0, 2500]), (2560, 16, [900, 1, 0, 2500]), (2560, 144, [900, 3000])])
def test_in_8_bits_large(N, K, counts):
    rows, E, g = sum(counts), len(counts), gen(3)
    A = torch.randint(-128, 128, (rows, K), generator=g, device=DEV, dtype=torch.int8)
    B = torch.randint(-128, 128, (E, N, K), generator=g, device=DEV, dtype=torch.int8)
    sa, sb = torch.exp(torch.randn(rows, generator=g, device=DEV)), torch.exp(torch.randn((E, N), generator=g, device=DEV))
    C = torch.full((rows, N), OUTSIDE, device=DEV)
    o = offsets_of(counts)
    t3.t3_gemm_grouped_i8(t3.grouped(rows, E, N, K), device(o), A, sa, B, sb, C)
    for e, (a, b) in enumerate(spans(o, rows)):
        close(C[a:b], *product8(A[a:b], sa[a:b], B[e], sb[e]))


# ------------------------------------------------------------------ the gradient of the weights

def check_wgrad(counts, first, behind, N, K, kn, add, integers, pads=(0, 0, 0, 0)):
    g = gen(N + K + len(counts))
    rows, E = first + sum(counts) + behind, len(counts)
    o = offsets_of(counts, first)
    pa, pc, pb, ps = pads
    A, dC = bf16(g, rows, K + pa), bf16(g, rows, N + pc)
    if integers:
        A, dC = (A * 2).round().clamp(-8, 8), (dC * 2).round().clamp(-8, 8)
    for t in (A, dC):
        t[:first], t[o[-1]:] = float("nan"), float("inf")
    r, c = (K, N) if kn else (N, K)
    flat = torch.full((E * (r * (c + pb) + ps),), OUTSIDE, device=DEV)
    if add:
        flat = torch.randint(-50, 51, flat.shape, generator=g, device=DEV).float()
    old = flat.clone()
    stride = r * (c + pb) + ps
    p = t3.grouped(rows, E, N, K, b_layout=t3.T3_B_KN if kn else t3.T3_B_NK, lda=K + pa, ldc=N + pc, ldb=c + pb, stride_b=stride,
                   flags=t3.T3_GROUPED_ACCUMULATE if add else 0)
    t3.t3_gemm_grouped_wgrad(p, device(o), A, dC, flat)
    torch.cuda.synchronize()
    for e, (a, b) in enumerate(spans(o, rows)):
        block = lambda f: f[e * stride:e * stride + r * (c + pb)].view(r, c + pb)
        x, d = A[a:b, :K], dC[a:b, :N]
        left, right = (x, d) if kn else (d, x)
        want, bound = left.double().t() @ right.double(), sum_bound(left.t(), right)
        if add:
            before = block(old)[:, :c].double()
            want, bound = want + before, bound + 2 * HALF * MORE * (before.abs() + want.abs() + bound)
        if integers:
            assert torch.equal(block(flat)[:, :c].double(), want), (e, a, b)
        else:
            close(block(flat)[:, :c], want, bound)
        assert torch.equal(block(flat)[:, c:], block(old)[:, c:])
        assert torch.equal(flat[e * stride + r * (c + pb):(e + 1) * stride], old[e * stride + r * (c + pb):(e + 1) * stride])


@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("case", range(len(GROUPS)))
def test_wgrad(case, layout):
    counts, first, behind = GROUPS[case]
    for i, (N, K) in enumerate([(8, 8), (40, 72), (264, 136), (520, 264)]):
        if N * K * len(counts) > 1.5e7:
            continue
        print(counts[:8], first, behind, N, K, flush=True)
        check_wgrad(counts, first, behind, N, K, layout == "kn", bool((case + i) % 2), i % 2 == 0)


@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("add", [False, True])
def test_wgrad_strides_and_lengths(layout, add):
    check_wgrad([1, 63, 64, 65, 0, 127, 128, 129, 191, 193], 2, 1, 136, 264, layout == "kn", add, False, pads=(8, 16, 4, 12))
    check_wgrad([300, 0, 1, 2000], 2, 1, 1032, 520, layout == "kn", add, True, pads=(8, 16, 4, 12))


@pytest.mark.parametrize("N,K,counts", [(2048, 1024, [700, 300, 0, 1500]), (1280, 2560, [4000, 60])])
def test_wgrad_large(N, K, counts):
    check_wgrad(counts, 0, 3, N, K, False, False, True)
    check_wgrad(counts, 0, 3, N, K, True, True, False)


def test_wgrad_of_more_tiles_than_a_launch_has_is_refused():
    N, K, E = 1 << 24, 8, 64
    assert grouped_tile(True, True, N, K, 4, E, wide_ok=False)[0] is False     # (rows of 32 MB)
    dB = torch.empty((E, N, K), device=DEV)
    with pytest.raises(t3.T3Error) as e:
        t3.t3_gemm_grouped_wgrad(t3.grouped(4, E, N, K), device([0] * E + [4]), torch.zeros((4, K), dtype=torch.bfloat16, device=DEV),
                                 torch.zeros((4, N), dtype=torch.bfloat16, device=DEV), dB)
    assert e.value.status == t3.T3_ERR_UNSUPPORTED


# several rounds of tiles, whose groups the launch takes by their lengths: like ones, empty ones, one that has nearly all rows, and more than it sorts
BY_LENGTH = [([125] * 64, 1024, 1024), ([0] * 20 + [1, 5000, 2] + [64] * 10, 2048, 1024), ([7 * i % 190 for i in range(17)], 1288, 1032),
             (list(range(65)), 2048, 2048), ([90 - i for i in range(64)], 1024, 768), ([0] * 17, 1288, 1032)]


@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("case", range(len(BY_LENGTH)))
def test_wgrad_of_several_rounds(case, layout):
    counts, N, K = BY_LENGTH[case]
    M, n = (K, N) if layout == "kn" else (N, K)
    wide, tm, tn, _ = grouped_tile(True, True, M, n, sum(counts) + 6, len(counts))
    assert wide and len(counts) * -(-M // tm) * -(-n // tn) > 256
    check_wgrad(counts, 4, 2, N, K, layout == "kn", bool(case % 2), case % 3 == 0)


# ------------------------------------------------------------------ together

def test_layer_of_experts_and_its_gradients():
    """Forward, gradient to the rows and gradient of the weights of one layer against autograd in 64 bits, and against differences
    of the forward product."""
    counts, N, K = [70, 0, 129, 1], 192, 320
    rows, E, g, o = sum(counts), len(counts), gen(9), offsets_of(counts)
    x, w, d = bf16(g, rows, K), bf16(g, E, N, K), bf16(g, rows, N)
    C, dx, dw = (torch.empty(s, device=DEV) for s in ((rows, N), (rows, K), (E, N, K)))
    off = device(o)
    t3.t3_gemm_grouped(t3.grouped(rows, E, N, K), off, x, w, C)
    t3.t3_gemm_grouped(t3.grouped(rows, E, K, N, b_layout=t3.T3_B_KN), off, d, w, dx)      # w is stored N x K
    t3.t3_gemm_grouped_wgrad(t3.grouped(rows, E, N, K), off, x, d, dw)
    x64, w64 = x.double().requires_grad_(), w.double().requires_grad_()
    out = torch.cat([x64[a:b] @ w64[e].t() for e, (a, b) in enumerate(spans(o, rows))])
    (out * d.double()).sum().backward()
    for e, (a, b) in enumerate(spans(o, rows)):
        close(C[a:b], out[a:b].detach(), sum_bound(x[a:b], w[e].t()))
        close(dx[a:b], x64.grad[a:b], sum_bound(d[a:b], w[e]))
        close(dw[e], w64.grad[e], sum_bound(d[a:b].t(), x[a:b]))
    # the product is linear in w: its change under a step of 1 in one weight is the gradient's element, whatever the step
    for e, n, k in [(0, 5, 300), (2, 191, 0), (3, 0, 7), (1, 3, 3)]:
        w2, C2 = w.clone(), torch.empty_like(C)
        w2[e, n, k] = float(w[e, n, k]) + 1.0
        t3.t3_gemm_grouped(t3.grouped(rows, E, N, K), off, x, w2, C2)
        step = float(w2[e, n, k].double() - w[e, n, k].double())
        a, b = spans(o, rows)[e]
        slack = float((sum_bound(x[a:b], w[e].t()).sum(0)[n] + sum_bound(x[a:b], w2[e].t()).sum(0)[n]) * d[a:b, n].double().abs().max()) if b > a else 0.0
        diff = float(((C2 - C).double() * d.double()).sum())
        assert abs(diff - step * float(dw[e, n, k])) <= slack + float(sum_bound(d[a:b].t(), x[a:b])[n, k]) * abs(step)


def test_experts_served_in_8_bits():
    counts, N, K = [3, 0, 1, 40, 7], 260, 528
    rows, E, g, o = sum(counts) + 4, len(counts), gen(4), offsets_of(counts)
    x, w = torch.randn((rows, K), generator=g, device=DEV), bf16(g, E, N, K)
    qx, sx = torch.empty((rows, K), dtype=torch.int8, device=DEV), torch.empty(rows, device=DEV)
    qw, sw = torch.empty((E, N, K), dtype=torch.int8, device=DEV), torch.empty((E, N), device=DEV)
    C = torch.full((rows, N), OUTSIDE, device=DEV)
    t3.t3_quant_rows(E * N, K, w, qw, sw)
    t3.t3_quant_rows(rows, K, x, qx, sx)
    t3.t3_gemm_grouped_i8(t3.grouped(rows, E, N, K), device(o), qx, sx, qw, sw, C)
    want_q, want_s = rows8(x.double().cpu().numpy())
    assert (qx.cpu().numpy() == want_q).all() and (sx.cpu().numpy() == want_s).all()
    for e, (a, b) in enumerate(spans(o, rows)):
        close(C[a:b], *product8(qx[a:b], sx[a:b], qw[e], sw[e]))
    assert bool((C[o[-1]:] == OUTSIDE).all())


def test_same_inputs_same_bits_on_other_streams_and_in_a_graph_with_new_offsets():
    N, K, E, rows = 520, 640, 6, 400
    g = gen(8)
    x, w, d = bf16(g, rows, K), bf16(g, E, N, K), bf16(g, rows, N)
    routes = [[100, 0, 50, 200, 1, 49], [0, 0, 400, 0, 0, 0], [66, 67, 66, 67, 67, 60]]
    off = device(offsets_of(routes[0]))

    def buffers():
        return torch.zeros((rows, N), device=DEV), torch.zeros((rows, K), device=DEV), torch.zeros((E, N, K), device=DEV)

    def step(C, dx, dw, offsets, stream=None):
        t3.t3_gemm_grouped(t3.grouped(rows, E, N, K), offsets, x, w, C, stream=stream)
        t3.t3_gemm_grouped(t3.grouped(rows, E, K, N, b_layout=t3.T3_B_KN), offsets, d, w, dx, stream=stream)
        t3.t3_gemm_grouped_wgrad(t3.grouped(rows, E, N, K), offsets, x, d, dw, stream=stream)

    want = []
    for r in routes:
        b = buffers()
        step(*b, device(offsets_of(r)))
        torch.cuda.synchronize()
        want.append([t.clone() for t in b])
    all_off, streams, got = [device(offsets_of(r)) for r in routes], [torch.cuda.Stream() for _ in routes], [buffers() for _ in routes]
    torch.cuda.synchronize()
    for _ in range(3):
        for o, st, b in zip(all_off, streams, got):
            step(*b, o, stream=st)
    torch.cuda.synchronize()
    for b, ref in zip(got, want):
        assert all(torch.equal(t, r) for t, r in zip(b, ref))
    b = buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*b, off)
    for i in (1, 2, 0, 1):
        off.copy_(all_off[i])
        for t in b:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, r) for t, r in zip(b, want[i]))


# ------------------------------------------------------------------ a rank that got no rows

@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("N,K,E,wide", [(24, 40, 3, False), (1032, 520, 9, True)])
def test_wgrad_of_no_rows(N, K, E, wide, add, layout):
    """Tensors of no rows have no address; all gradients are zeros, or unchanged where they are added to."""
    kn = layout == "kn"
    M, n = (K, N) if kn else (N, K)
    assert grouped_tile(True, True, M, n, 0, E)[0] == wide
    A, dC = (torch.empty((0, c), dtype=torch.bfloat16, device=DEV) for c in (K, N))
    assert A.data_ptr() == 0 and dC.data_ptr() == 0
    dB = torch.randn((E + 1, M, n), generator=gen(N), device=DEV)
    old = dB.clone()
    p = t3.grouped(0, E, N, K, b_layout=t3.T3_B_KN if kn else t3.T3_B_NK, flags=t3.T3_GROUPED_ACCUMULATE if add else 0)
    t3.t3_gemm_grouped_wgrad(p, device([0] * (E + 1)), A, dC, dB)
    torch.cuda.synchronize()
    assert torch.equal(dB[:E], old[:E] if add else torch.zeros_like(old[:E])) and torch.equal(dB[E], old[E])


def test_layer_of_no_rows_and_products_of_no_contraction():
    E, N, K, off = 3, 64, 128, device([0] * 4)
    x, y, c = (torch.empty((0, w), dtype=d, device=DEV) for w, d in ((K, torch.bfloat16), (N, torch.bfloat16), (N, torch.float32)))
    q, s = torch.empty((0, K), dtype=torch.int8, device=DEV), torch.empty(0, device=DEV)
    w, w8, sw = bf16(gen(0), E, N, K), torch.ones((E, N, K), dtype=torch.int8, device=DEV), torch.ones((E, N), device=DEV)
    t3.t3_quant_rows(0, K, x, q, s)
    t3.t3_gemm_grouped(t3.grouped(0, E, N, K), off, x, w, c)
    t3.t3_gemm_grouped(t3.grouped(0, E, K, N, b_layout=t3.T3_B_KN), off, y, w, torch.empty((0, K), device=DEV))
    t3.t3_gemm_grouped_i8(t3.grouped(0, E, N, K), off, q, s, w8, sw, c)
    t3.t3_gemm_i8(t3.problem(0, N, K, 1, 0), q, s, w8, sw, c)
    # no contraction: products of zeros, of operands that have no address
    C = torch.full((6, N), OUTSIDE, device=DEV)
    for i8 in (False, True):
        C.fill_(OUTSIDE)
        none, one = torch.empty((6, 0), dtype=torch.int8 if i8 else torch.bfloat16, device=DEV), torch.ones(max(6, E * N), device=DEV)
        if i8:
            t3.t3_gemm_grouped_i8(t3.grouped(6, E, N, 0), device([1, 2, 2, 5]), none, one, none, one, C)
        else:
            t3.t3_gemm_grouped(t3.grouped(6, E, N, 0), device([1, 2, 2, 5]), none, none, C)
        torch.cuda.synchronize()
        assert bool((C[1:5] == 0.0).all()) and bool((C[:1] == OUTSIDE).all()) and bool((C[5:] == OUTSIDE).all())
    C.fill_(OUTSIDE)
    t3.t3_gemm_i8(t3.problem(6, N, 0, 1, 0), none, one, none, one, C)
    s0 = torch.full((3,), OUTSIDE, device=DEV)
    t3.t3_quant_rows(2, 0, torch.empty((2, 0), dtype=torch.bfloat16, device=DEV), torch.empty((2, 0), dtype=torch.int8, device=DEV), s0)
    torch.cuda.synchronize()
    assert bool((C == 0.0).all()) and s0.tolist() == [0.0, 0.0, OUTSIDE]


@pytest.mark.parametrize("ldb,wide", [(1 << 24, True), (1 << 25, False), (1 << 26, False)])
def test_short_contraction_of_far_rows(ldb, wide):
    """Eight k-rows of B far from one another: the others of a slab are zeros, not rows that are there (an infinity times A's zeros would be NaN)."""
    K, counts = 8, [700, 900, 1, 450, 0, 1300]
    N, rows, g, o = 2600, sum(counts), gen(1), offsets_of(counts)
    assert grouped_wide_fits(True, K, K, ldb, N) == wide and grouped_tile(False, True, rows, N, K, len(counts))[0]
    A = torch.randint(1, 9, (rows, K), generator=g, device=DEV).to(torch.bfloat16)
    B = torch.zeros((K, ldb), dtype=torch.bfloat16, device=DEV)
    B[:, :N] = torch.randint(-8, 9, (K, N), generator=g, device=DEV).to(torch.bfloat16)
    B[0, 5::64], B[7, 9::64] = float("inf"), -float("inf")
    C = torch.full((rows, N), OUTSIDE, device=DEV)
    t3.t3_gemm_grouped(t3.grouped(rows, len(counts), N, K, b_layout=t3.T3_B_KN, ldb=ldb, stride_b=0), device(o), A, B, C)
    assert torch.equal(C.double(), A.double() @ B[:, :N].double())


# ------------------------------------------------------------------ more workgroups than one launch has lanes for

def test_forward_of_several_launches():
    counts = [1, 0, 2] * 60 + [1] * 75
    N, K, E, rows = 4194300, 8, len(counts), sum(counts)
    wide, tm, tn, _ = grouped_tile(False, False, rows, N, K, E, wide_ok=grouped_wide_fits(False, K, K, K, N))
    assert not wide and sum(-(-n // tm) for n in counts) * -(-N // tn) > 1 << 24
    g, o = gen(4), offsets_of(counts)
    A, B = (torch.randint(-8, 9, (n, K), generator=g, device=DEV).to(torch.bfloat16) for n in (rows, N))
    C = torch.full((rows, N), OUTSIDE, device=DEV)
    t3.t3_gemm_grouped(t3.grouped(rows, E, N, K, stride_b=0), device(o), A, B, C)
    for c in range(0, N, 1 << 18):                    # (whole numbers: exact)
        assert torch.equal(C[:, c:c + (1 << 18)], A.float() @ B[c:c + (1 << 18)].float().t()), c


@pytest.mark.parametrize("add", [False, True])
def test_wgrad_of_several_launches(add):
    N, K, E = 1 << 23, 8, 64
    M, n, counts = N, K, [0] * 30 + [3] + [0] * 32 + [1]
    wide, tm, tn, _ = grouped_tile(True, True, M, n, 4, E, wide_ok=False)
    assert not wide and E * (M // tm) >= 1 << 24 > E * (M // 64)
    g, o = gen(5), offsets_of(counts)
    A, dC = (torch.randint(-8, 9, (4, w), generator=g, device=DEV).to(torch.bfloat16) for w in (K, N))
    dB = torch.full((E, N, K), 3.0, device=DEV)
    t3.t3_gemm_grouped_wgrad(t3.grouped(4, E, N, K, flags=t3.T3_GROUPED_ACCUMULATE if add else 0), device(o), A, dC, dB)
    for e, (a, b) in enumerate(spans(o, 4)):
        assert torch.equal(dB[e], dC[a:b].float().t() @ A[a:b].float() + (3.0 if add else 0.0)), e


# ------------------------------------------------------------------ timeline

@pytest.mark.parametrize("counts,cut", ROUNDS)
@pytest.mark.parametrize("call", ["nk", "kn", "8 bits"])
def test_timeline_of_two_launches(call, counts, cut):
    """Every tile leaves four readings, those of the last round that are done in quarters behind the full rounds; results are the same."""
    N, K, rows, E, kn = 6144, 1024, sum(counts), len(counts), call == "kn"
    T, left = quarters(counts, N, (256, 256))
    assert left == cut and grouped_tile(False, kn, rows, N, K, E)[1:] == (256, 256, True)
    g, off = gen(11), device(offsets_of(counts))
    p = t3.grouped(rows, E, N, 2 * K if call == "8 bits" else K, b_layout=t3.T3_B_KN if kn else t3.T3_B_NK)
    if call == "8 bits":
        A, B = (torch.randint(-128, 128, (n, 2 * K), generator=g, device=DEV, dtype=torch.int8) for n in (rows, E * N))
        sa, sb = torch.ones(rows, device=DEV), torch.ones(E * N, device=DEV)
    else:
        A, B = bf16(g, rows, K), bf16(g, E, *((K, N) if kn else (N, K)))

    def run(C):
        if call == "8 bits":
            t3.t3_gemm_grouped_i8(p, off, A, sa, B, sb, C)
        else:
            t3.t3_gemm_grouped(p, off, A, B, C)
        torch.cuda.synchronize()
        return C

    want = run(torch.zeros((rows, N), device=DEV))
    items = t3.T3_TIMELINE_ITEMS
    st = torch.full((520, items, 4), -1, dtype=torch.int64, device=DEV)
    t3.t3_timeline(st)
    try:
        got = run(torch.zeros((rows, N), device=DEV))
    finally:
        t3.t3_timeline(None)
    assert torch.equal(got, want)
    st = st.cpu()
    taken = (st != -1).all(dim=2)
    assert torch.equal(taken, (st != -1).any(dim=2))
    rounds, last = (T - left) // 256, (T - left) % 256
    assert bool(taken[:256, :rounds].all()) and int(taken[256:, :rounds].sum()) == 0
    if left:
        # quarters of the last tiles that hold rows (N is whole tiles): half of a group's last tile may be none
        assert last == 0 and 2 * left <= int(taken[:, rounds].sum()) <= 4 * left and int(taken[:, rounds + 1:].sum()) == 0
    else:
        assert int(taken[:, rounds].sum()) == last and int(taken[:, rounds + 1:].sum()) == 0
    for w in range(520):
        readings = st[w][taken[w]].flatten().tolist()
        assert readings == sorted(readings), w


# ------------------------------------------------------------------ more groups than a wavefront has lanes, on the largest tiles

# groups, the lengths' modulus, tiles of the last round that are done in quarters (of the last groups)
MANY = [(65, 487, 124), (100, 521, 96), (128, 509, 40), (129, 509, 48), (193, 401, 28), (256, 509, 12)]


@pytest.mark.parametrize("layout", ["nk", "kn", "8 bits"])
@pytest.mark.parametrize("E,mod,cut", MANY)
def test_more_than_64_groups_on_the_largest_tiles(E, mod, cut, layout):
    counts = [(37 * i * i + 11 * i) % mod for i in range(E)]
    N, K, rows, kn = 1024, 1024, sum(counts) + 3, layout == "kn"
    assert counts[0] == 0 and grouped_tile(False, kn, rows, N, K, E) == (True, 256, 256, True)
    assert quarters(counts, N, (256, 256))[1] == cut
    if layout != "8 bits":
        check_forward(counts, 1, 2, N, K, kn, integers=E % 2 == 0)
        return
    g, o = gen(E), offsets_of(counts, 1)
    A = torch.randint(-128, 128, (rows, 2 * K), generator=g, device=DEV, dtype=torch.int8)
    B = torch.randint(-128, 128, (E, N, 2 * K), generator=g, device=DEV, dtype=torch.int8)
    sa, sb = torch.exp(torch.randn(rows, generator=g, device=DEV)), torch.exp(torch.randn((E, N), generator=g, device=DEV))
    C = torch.full((rows, N), OUTSIDE, device=DEV)
    t3.t3_gemm_grouped_i8(t3.grouped(rows, E, N, 2 * K), device(o), A, sa, B, sb, C)
    for e, (a, b) in enumerate(spans(o, rows)):
        close(C[a:b], *product8(A[a:b], sa[a:b], B[e], sb[e]))
    assert bool((C[:1] == OUTSIDE).all()) and bool((C[o[-1]:] == OUTSIDE).all())
