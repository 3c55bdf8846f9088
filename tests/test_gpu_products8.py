"""Rows in 8 bits (t3_quant_rows) and products of them (t3_gemm_i8, t3_gemm_rs_fused_i8) on the GPU against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2401_16677_amd import binding as t3
from products import HALF, MORE, close, product8, rows8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def int8(g, rows, cols, ld=None):
    t = torch.randint(-128, 128, (max(rows, 1), cols if ld is None else ld), generator=g, device=DEV, dtype=torch.int8)
    return t


def scales(g, n):
    return torch.exp(torch.randn(max(n, 1), generator=g, device=DEV))


# ------------------------------------------------------------------ rows

def quantised(x, rows, cols, ldq=None):
    ldq = cols if ldq is None else ldq
    q = torch.full((rows + 1, max(ldq, 8)), 99, dtype=torch.int8, device=DEV)
    s = torch.full((rows + 1,), 7.0, device=DEV)
    t3.t3_quant_rows(rows, cols, x, q, s, ldx=x.shape[1], ldq=q.shape[1])
    torch.cuda.synchronize()
    assert bool((q[rows:] == 99).all()) and bool((q[:, cols:] == 99).all()) and float(s[rows]) == 7.0
    return q[:rows, :cols].cpu().numpy(), s[:rows].cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,pad", [(1, 8, 0), (3, 24, 8), (5, 512, 0), (257, 136, 16), (4, 4096, 0), (2, 4104, 0), (3, 16384, 8),
                                           (2, 16392, 0), (1, 40000, 0), (1000, 1152, 0)])
def test_rows(dtype, rows, cols, pad):
    g = gen(rows * 131 + cols)
    x = (torch.randn((rows, cols + pad), generator=g, device=DEV) * torch.exp(4 * torch.randn((rows, 1), generator=g, device=DEV))).to(dtype)
    x[:, cols:] = 1e30                              # not of the row
    if rows > 2:
        x[1] = 0.0
    q, s = quantised(x, rows, cols, cols + pad)
    want_q, want_s = rows8(x[:, :cols].double().cpu().numpy())
    assert np.array_equal(q, want_q) and np.array_equal(s, want_s)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("top", [127.0, 254.0, 2.0 ** -133, 127 * 2.0 ** -130, 3.0e38, 1.0])
def test_rows_borders(dtype, top):
    """Quotients that are halves, or as near to one as the type has numbers; magnitudes whose inverse no float holds."""
    unit = top / 127.0
    x = torch.tensor([[top, -top] + [(k + 0.5) * unit * (1 if k % 2 else -1) for k in range(0, 126)]], dtype=torch.float64).to(dtype)
    near = [x] + [torch.nextafter(x.float(), torch.full_like(x, t, dtype=torch.float32)).to(dtype) for t in (-np.inf, np.inf)] \
        if dtype == torch.float32 else [x, x * 0.5, x * 0.998046875]
    x = torch.cat(near).clamp(-top, top).to(DEV)
    q, s = quantised(x, x.shape[0], x.shape[1])
    want_q, want_s = rows8(x.double().cpu().numpy())
    assert np.array_equal(q, want_q) and np.array_equal(s, want_s)


def test_rows_of_several_launches():
    """More rows than a launch has wavefronts for, and rows without columns."""
    rows, g = (1 << 25) + 5, gen(2)
    x = torch.randn((rows, 8), generator=g, device=DEV).to(torch.bfloat16)
    q, s = torch.full((rows + 1, 8), 99, dtype=torch.int8, device=DEV), torch.full((rows + 1,), 7.0, device=DEV)
    t3.t3_quant_rows(rows, 8, x, q, s)
    for at in (slice(0, 9), slice((1 << 25) - 9, rows)):
        want_q, want_s = rows8(x[at].double().cpu().numpy())
        assert np.array_equal(q[at].cpu().numpy(), want_q) and np.array_equal(s[at].cpu().numpy(), want_s)
    assert bool((q[:rows].abs().amax(1) == 127).all()) and bool((q[rows] == 99).all()) and float(s[rows]) == 7.0
    t3.t3_quant_rows(3, 0, x, q, s, ldx=8, ldq=8)
    assert s[:4].tolist() == [0.0, 0.0, 0.0, float(rows8(x[3:4].double().cpu().numpy())[1][0])]


def test_rows_that_are_no_numbers():
    x = torch.ones((5, 72), device=DEV)
    x[1, 3], x[2, 70], x[3, 0], x[4] = float("nan"), float("inf"), float("-inf"), 0.0
    for y in (x, x.to(torch.bfloat16)):
        q, s = quantised(y, 5, 72)
        assert (q[0] == 127).all() and (q[1:] == 0).all()
        assert np.isnan(s[1:4]).all() and s[4] == 0.0


# ------------------------------------------------------------------ the plain product

SHAPES = [(1, 4, 16), (1, 1200, 1536), (3, 20, 48), (16, 516, 1040), (17, 100, 272), (33, 64, 64), (64, 260, 128), (100, 1000, 2000), (130, 772, 640),
          (300, 1028, 1168), (515, 2052, 336), (1000, 600, 4112), (2048, 2560, 512), (257, 8200, 1536), (4100, 1540, 768),
          (2100, 2564, 112), (2100, 2564, 128), (3000, 5140, 16), (2100, 2564, 144)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(M, N, K):
    g = gen(M + N + K)
    a, b, sa, sb = int8(g, M, K), int8(g, N, K), scales(g, M), scales(g, N)
    c = torch.full((M + 1, N), 5.0, device=DEV)
    t3.t3_gemm_i8(t3.problem(M, N, K, 1, 0), a, sa, b, sb, c)
    torch.cuda.synchronize()
    close(c[:M], *product8(a, sa, b, sb))
    assert bool((c[M] == 5.0).all())
    # with whole scales the sums below 2^24 come out as they are
    one = torch.ones(max(M, N), device=DEV)
    small_a, small_b = a % 8, b % 8
    t3.t3_gemm_i8(t3.problem(M, N, K, 1, 0), small_a, one, small_b, one, c)
    assert torch.equal(c[:M].double(), small_a.double() @ small_b.double().t())


@pytest.mark.parametrize("M,N,K,tp", [(40, 96, 80, 4), (300, 1056, 400, 2), (700, 2112, 1200, 8)])
def test_product_strides_chunks_and_columns_beside(M, N, K, tp):
    g = gen(5)
    a, b, sa, sb = int8(g, M, K, K + 48), int8(g, N, K, K + 16), scales(g, M + 5)[5:], scales(g, N + 3)[3:]
    c = torch.full((M, N + 12), 5.0, device=DEV)
    t3.t3_gemm_i8(t3.problem(M, N, K, tp, tp - 1, lda=K + 48, ldb=K + 16, ldc=N + 12), a, sa, b, sb, c)
    torch.cuda.synchronize()
    close(c[:, :N], *product8(a[:, :K], sa, b[:, :K], sb))
    assert bool((c[:, N:] == 5.0).all())


# a last round of at most half the workgroups of 256 x 192 and 256 x 256: its tiles in halves of K
@pytest.mark.parametrize("M,N,K", [(1000, 16640, 1040), (2040, 10240, 2064), (1000, 20484, 1040)])
def test_product_of_a_split_last_round(M, N, K):
    g = gen(K)
    a, b, sa, sb = int8(g, M, K), int8(g, N, K), scales(g, M), scales(g, N)
    c, p = torch.full((M, N), 5.0, device=DEV), t3.problem(M, N, K, 1, 0)
    want, bound = product8(a, sa, b, sb)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t3.t3_gemm_i8(p, a, sa, b, sb, c)
    for i in range(4):                              # eager and replayed calls in turn, with the same flags between the halves
        c.fill_(5.0)
        if i % 2:
            graph.replay()
        else:
            t3.t3_gemm_i8(p, a, sa, b, sb, c)
        torch.cuda.synchronize()
        close(c, want, bound)


def test_product_at_its_limits():
    """The largest sum of the longest K, no K, no rows, scales of zero and of no number."""
    K = 131056
    a, b = torch.full((2, K), -128, dtype=torch.int8, device=DEV), torch.full((4, K), -128, dtype=torch.int8, device=DEV)
    one, c = torch.ones(4, device=DEV), torch.zeros((2, 4), device=DEV)
    t3.t3_gemm_i8(t3.problem(2, 4, K, 1, 0), a, one, b, one, c)
    assert bool((c == float(K * 16384)).all())
    t3.t3_gemm_i8(t3.problem(2, 4, 0, 1, 0), a, one, b, one, c)
    assert bool((c == 0.0).all())
    c.fill_(3.0)
    t3.t3_gemm_i8(t3.problem(0, 4, 16, 1, 0), a, one, b, one, c)
    t3.t3_gemm_i8(t3.problem(2, 4, 16, 1, 0, 128, 128, tile_begin=1, tile_limit=1), a, one, b, one, c)      # (an empty range)
    assert bool((c == 3.0).all())
    s = torch.tensor([0.0, float("nan")], device=DEV)
    t3.t3_gemm_i8(t3.problem(2, 4, 64, 1, 0), a, s, b, one, c)
    assert bool((c[0] == 0.0).all()) and bool(c[1].isnan().all())


# ------------------------------------------------------------------ into the ring's partials

FUSED = [(24, 1152, 1152, 16, 9, 0, (0, 0)), (100, 320, 400, 4, 3, t3.T3_FLAG_FWD_DIRECT, (128, 128)),
         (257, 1040, 640, 2, 0, t3.T3_FLAG_FWD_BF16 | t3.T3_FLAG_FWD_DIRECT, (0, 0)), (520, 2144, 336, 4, 1, t3.T3_FLAG_FWD_BF16, (256, 128)),
         (1000, 2128, 1072, 4, 2, t3.T3_FLAG_STEP0_STORE_ONLY, (128, 256)), (2040, 5120, 1040, 5, 2, t3.T3_FLAG_FWD_DIRECT, (256, 256)),
         (1100, 3200, 576, 8, 7, t3.T3_FLAG_FWD_DIRECT | t3.T3_FLAG_STEP0_STORE_ONLY, (0, 0)), (700, 1504, 2000, 2, 1, 0, (0, 0)), (64, 64, 32, 1, 0, 0, (0, 0)),
         (1000, 16640, 1040, 5, 3, t3.T3_FLAG_FWD_DIRECT, (0, 0)), (2040, 10240, 2064, 8, 0, 0, (256, 256)),
         (2000, 4096, 112, 4, 1, t3.T3_FLAG_FWD_DIRECT, (256, 256)), (2300, 4256, 128, 8, 5, 0, (0, 0))]


def fused_case(M, N, K, tp, seed=3):
    g = gen(seed)
    a, b, sa, sb = int8(g, M, K), int8(g, N, K), scales(g, M) * 0.01, scales(g, N) * 0.01
    return a, b, sa, sb, torch.randn((M, N), generator=g, device=DEV) * 30.0


def check_ring(M, N, tp, rank, flags, tile, got_R, got_fwd, track, inc, C, bound, oracle):
    W, bf16 = N // tp, bool(flags & t3.T3_FLAG_FWD_BF16)
    order, own = t3.t3_chunk_order(tp, rank)
    for i, c in enumerate(order):
        cols = slice(c * W, (c + 1) * W)
        old = inc[:, cols].double()
        first = i == 0 and flags & t3.T3_FLAG_STEP0_STORE_ONLY
        want = C[:, cols] + (0.0 if first else old)
        # two additions round numbers of at most |incoming| + |product| and what has been added so far
        lim = bound[:, cols] + 2 * HALF * MORE * (old.abs() * (not first) + C[:, cols].abs() + bound[:, cols])
        if c != own:
            close(got_fwd[i], want, lim + ((want.abs() + lim) * 2.0 ** -8 if bf16 else 0.0))
        if c == own or not flags & t3.T3_FLAG_FWD_DIRECT:
            close(got_R[:, cols], want, lim)
        else:
            assert torch.equal(got_R[:, cols], inc[:, cols])
    tr = t3.read_track(track, tp)
    tm, tn = tile if tile != (0, 0) else t3.t3_default_tile(t3.problem(M, N, 64, tp, rank))
    assert (tr["counter"] == oracle.tiles_per_chunk(M, N, tp, tm, tn)).all() and (tr["ready"] == 1).all()
    assert set(tr["queue"][:tp - 1].tolist()) == set(order[:-1]) and tr["queue_len"] == tp - 1 and tr["error"] == 0


@pytest.mark.parametrize("M,N,K,tp,rank,flags,tile", FUSED)
def test_fused(M, N, K, tp, rank, flags, tile, oracle):
    a, b, sa, sb, inc = fused_case(M, N, K, tp)
    R, track = inc.clone(), torch.zeros(t3.t3_track_words(tp), dtype=torch.int32, device=DEV)
    fwd = torch.full((max(tp - 1, 1), M, N // tp), -7.0, dtype=torch.bfloat16 if flags & t3.T3_FLAG_FWD_BF16 else torch.float32, device=DEV)
    p = t3.problem(M, N, K, tp, rank, *tile, flags=flags)
    t3.t3_track_reset(tp, track)
    C, bound = product8(a, sa, b, sb)
    for _ in range(2):                              # the tracker's other bank too
        R.copy_(inc)
        t3.t3_gemm_rs_fused_i8(p, a, sa, b, sb, R, fwd, track)
        torch.cuda.synchronize()
        check_ring(M, N, tp, rank, flags, tile, R, fwd, track, inc, C, bound, oracle)


def test_fused_ring_step_by_step(oracle):
    """One call per ring step: chunks become ready one by one, and the sum of the calls is the whole call."""
    M, N, K, tp, rank, tile = 300, 1024, 400, 4, 1, (128, 128)
    a, b, sa, sb, inc = fused_case(M, N, K, tp)
    track = torch.zeros(t3.t3_track_words(tp), dtype=torch.int32, device=DEV)
    R, fwd = inc.clone(), torch.zeros((tp - 1, M, N // tp), device=DEV)
    t3.t3_track_reset(tp, track)
    tpc = t3.t3_tiles_per_chunk(t3.problem(M, N, K, tp, rank, *tile))
    for s in range(tp):
        t3.t3_gemm_rs_fused_i8(t3.problem(M, N, K, tp, rank, *tile, tile_begin=s * tpc, tile_limit=(s + 1) * tpc), a, sa, b, sb, R, fwd, track)
        torch.cuda.synchronize()
        tr = t3.read_track(track, tp)
        assert [int(r) for r in tr["ready"]] == [int(c == (rank + s) % tp) for c in range(tp)]
    R1, fwd1 = inc.clone(), torch.zeros_like(fwd)
    t3.t3_gemm_rs_fused_i8(t3.problem(M, N, K, tp, rank, *tile), a, sa, b, sb, R1, fwd1, track)
    torch.cuda.synchronize()
    C, bound = product8(a, sa, b, sb)
    check_ring(M, N, tp, rank, 0, tile, R1, fwd1, track, inc, C, bound, oracle)
    lim = 2 * (bound + 2 * HALF * MORE * (inc.double().abs() + C.abs() + bound))
    close(R, R1.double(), lim)


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("M", [1, 5, 200, 900])
def test_layer_in_8_bits(M):
    """A row-parallel layer served in 8 bits: the all-reduced fp32 activations and the weights to 8 bits, the product of them."""
    N, K = 1028, 1040
    g = gen(M)
    x = torch.randn((M, K), generator=g, device=DEV)
    w = (torch.randn((N, K), generator=g, device=DEV) * K ** -0.5).to(torch.bfloat16)
    qx, qw = torch.empty((M, K), dtype=torch.int8, device=DEV), torch.empty((N, K), dtype=torch.int8, device=DEV)
    sx, sw, c = torch.empty(M, device=DEV), torch.empty(N, device=DEV), torch.empty((M, N), device=DEV)
    t3.t3_quant_rows(M, K, x, qx, sx)
    t3.t3_quant_rows(N, K, w, qw, sw)
    t3.t3_gemm_i8(t3.problem(M, N, K, 1, 0), qx, sx, qw, sw, c)
    close(c, *product8(qx, sx, qw, sw))
    # every value is off by at most half its row's unit: |error| <= sum |x| uw / 2 + |w| ux / 2 + ux uw / 4
    ux, uw = sx.double()[:, None], sw.double()[None, :]
    xs, ws = x.double().abs().sum(1, keepdim=True), w.double().abs().sum(1)[None, :]
    close(c, x.double() @ w.double().t(), MORE * (xs * uw / 2 + ws * ux / 2 + K * ux * uw / 4))


def test_calls_on_two_streams_and_in_a_graph():
    M, N, K = 260, 1540, 528
    g = gen(1)
    xs = [torch.randn((M, K), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2)]
    w, sw = int8(g, N, K), scales(g, N)

    def buffers():
        return torch.zeros((M, K), dtype=torch.int8, device=DEV), torch.zeros(M, device=DEV), torch.zeros((M, N), device=DEV)

    def layer(x, q, s, c, stream=None):
        t3.t3_quant_rows(M, K, x, q, s, stream=stream)
        t3.t3_gemm_i8(t3.problem(M, N, K, 1, 0), q, s, w, sw, c, stream=stream)

    want = []
    for x in xs:
        b = buffers()
        layer(x, *b)
        torch.cuda.synchronize()
        want.append([t.clone() for t in b])
    streams, got = [torch.cuda.Stream() for _ in xs], [buffers() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(4):
        for x, b, st in zip(xs, got, streams):
            layer(x, *b, stream=st)
    torch.cuda.synchronize()
    for b, ref in zip(got, want):
        assert all(torch.equal(t, r) for t, r in zip(b, ref))
    x, b = xs[0].clone(), buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(x, *b)
    for i in (0, 1, 0):
        x.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b[0], want[i][0]) and torch.equal(b[1], want[i][1])
        close(b[2], *product8(b[0], b[1], w, sw))
