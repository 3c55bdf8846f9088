"""The products in 8-bit integers and the products grouped by expert, as a list of measurable cases.

A case is one pass through the operators as a rank's program calls them:

  op = "linear8"  rows of activations quantised (t3_quant_rows), then t3_gemm_i8 with weights that were quantised once
  op = "ring8"    rows quantised, then t3_gemm_rs_fused_i8: the partial product added into the ring's partials chunk by chunk
  op = "experts"  t3_gemm_grouped: rows sorted by expert times each expert's weights, bf16; layout "nk" the forward product (B_e
                  stored N x K), "kn" the gradient to the rows (B_e stored K x N)
  op = "experts8" rows quantised, then t3_gemm_grouped_i8
  op = "wgrad"    t3_gemm_grouped_wgrad: the gradient of each expert's weights, in the layout of the weights; `add` into what is there

With `own` false the same is computed in elementary torch operations, products and sums in 32 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"


def _linear8(name, M, N, K):
    c = {"op": "linear8", "M": M, "N": N, "K": K}
    return c if name is None else {"name": name, **c}


def _ring8(name, M, N, K, tp, rank, tile, direct=True, fwd="fp32", step0=False):
    c = {"op": "ring8", "M": M, "N": N, "K": K, "tp": tp, "rank": rank, "tile_m": tile[0], "tile_n": tile[1],
         "direct": direct, "fwd": fwd, "step0_store": step0}
    return c if name is None else {"name": name, **c}


def _experts(name, op, rows, groups, N, K, layout="nk", spare=0, skew=0.0, add=False):
    c = {"op": op, "rows": rows, "groups": groups, "N": N, "K": K, "layout": layout, "spare": spare, "skew": skew, "add": add}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # one token against the output projection's slice of a GPT-3 sized layer served in 8 bits: launches and latency
        _linear8("i8_token_outproj", 1, 12288, 1536),
        # a serving batch of odd size against the FC-2 slice: bound by reading the weights
        _linear8("i8_decode_fc2", 37, 12288, 6144),
        # a prefill through the same FC-2 slice: matrix bound
        _linear8("i8_prefill_fc2", 4096, 12288, 6144),
        # a serving batch whose partial sums go round a ring of 16: weights and ring traffic, short K
        _ring8("i8_ring_decode", 24, 18432, 1152, 16, 9, (128, 128)),
        # a prefill's output projection with the ring's reduction: output traffic and products alike
        _ring8("i8_ring_outproj", 4096, 12288, 1536, 8, 3, (256, 256)),
        # one token routed to two of eight experts: two rows, two of the weights
        _experts("experts_token", "experts", 2, 8, 4096, 1024),
        # a prefill routed unevenly to 16 experts, rows to spare behind the last
        _experts("experts_prefill", "experts", 8192, 16, 5120, 1280, spare=64, skew=0.6),
        # training: the gradient to the rows of the same layer
        _experts("experts_dgrad", "experts", 8190, 16, 1280, 5120, layout="kn", skew=0.6),
        # training: the gradient of its weights
        _experts("experts_wgrad", "wgrad", 8190, 16, 5120, 1280, skew=0.6),
        # a small model's, few rows an expert, gradients of several micro-batches added up
        _experts("experts_wgrad_short", "wgrad", 301, 6, 520, 264, layout="kn", skew=0.3, add=True),
        # a serving batch spread over many experts: every expert's weights for a row or two
        _experts("experts_i8_decode", "experts8", 64, 32, 4096, 2048),
        # a long prefill in 8 bits
        _experts("experts_i8_prefill", "experts8", 16384, 8, 6144, 2048, skew=0.3),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: a token to a long prefill, narrow to wide, short to long K, one expert to many."""
    while True:
        op = rng.choice(("linear8", "linear8", "ring8", "experts", "experts", "experts8", "wgrad"))
        M = _logint(rng, 1, 16384)
        if op == "linear8":
            c = _linear8(None, M, _logint(rng, 64, 20480) // 4 * 4, _logint(rng, 128, 10240) // 16 * 16)
        elif op == "ring8":
            tp, fwd = rng.choice((2, 4, 8, 8, 16, 32)), rng.choice(("fp32", "fp32", "bf16"))
            col = 8 if fwd == "bf16" else 4
            W = max(col, _logint(rng, 1024, 20480) // tp // col * col)
            c = _ring8(None, M, W * tp, _logint(rng, 128, 10240) // 16 * 16, tp, rng.randrange(tp),
                       rng.choice(((128, 128), (256, 128), (256, 256))), rng.random() < 0.6, fwd, rng.random() < 0.25)
        else:
            layout = rng.choice(("nk", "nk", "kn")) if op != "experts8" else "nk"
            N = _logint(rng, 64, 8192) // 8 * 8
            K = _logint(rng, 64, 8192) // (64 if layout == "kn" and op == "experts" else 16) * (64 if layout == "kn" and op == "experts" else 16)
            c = _experts(None, op, M, _logint(rng, 1, 128), N, K, layout, rng.choice((0, 0, 17)), rng.choice((0.0, 0.3, 0.6, 1.2)),
                         op == "wgrad" and rng.random() < 0.3)
        w = work(c)
        if w["flops"] <= 6.1e11 and w["bytes"] <= 7e8 and c["N"] * c["K"] * c.get("groups", 1) <= 2.5e8:
            return c                                    # no dearer than the largest listed ones


# ------------------------------------------------------------------ inputs

def _rand(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _activations(g, rows, K):
    """Rows of their own size, a few channels much larger than the rest; a batch's last row is padding."""
    x = _rand(g, rows, K) * torch.exp(0.5 * _rand(g, rows, 1))
    x[:, :: max(1, K // 8)] *= 8.0
    if rows >= 8:
        x[-1] = 0.0
    return x.to(torch.bfloat16)


def _weights8(g, rows, K):
    """Weights of unit variance over K in 8 bits, a scale for each row, as a program loads them."""
    w = _rand(g, rows, K) * (K ** -0.5)
    top = w.abs().amax(dim=1, keepdim=True)
    return torch.round(w * (127.0 / top)).to(torch.int8), (top[:, 0] / 127.0).contiguous()


def _counts(case, seed):
    """Rows of each expert: drawn row by row, some experts likelier than others (some get none)."""
    g = torch.Generator()
    g.manual_seed(seed * 7919 + 11)
    p = torch.exp(case["skew"] * torch.randn(case["groups"], generator=g, dtype=torch.float64))
    to = torch.multinomial(p, case["rows"], replacement=True, generator=g)
    return torch.bincount(to, minlength=case["groups"]).tolist()


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    op, N, K = case["op"], case["N"], case["K"]
    st = {"op": op, "case": case}
    if op in ("linear8", "ring8"):
        M = case["M"]
        st["x"] = _activations(g, M, K)
        st["w"], st["sw"] = _weights8(g, N, K)
    if op == "linear8":
        st["C"] = torch.zeros((M, N), device=DEV)
    if op == "ring8":
        tp, bf16 = case["tp"], case["fwd"] == "bf16"
        st["R"] = _rand(g, M, N) * math.sqrt(tp - 1)
        st["fwd"] = torch.zeros((tp - 1, M, N // tp), dtype=torch.bfloat16 if bf16 else torch.float32, device=DEV)
        # the tracker's state: two banks of counters, flags and queue, then generation, error and words of the kernels' own
        st["track"] = torch.zeros(2 * (3 * tp + 2) + 2 + 256, dtype=torch.int32, device=DEV)
    if op in ("experts", "experts8", "wgrad"):
        rows, E, kn = case["rows"] + case["spare"], case["groups"], case["layout"] == "kn"
        st["counts"] = _counts(case, seed)
        st["offsets"] = torch.tensor([sum(st["counts"][:e]) for e in range(E + 1)], dtype=torch.int32).to(DEV)
        if op == "experts8":
            st["x"] = _activations(g, rows, K)
            st["w"], st["sw"] = _weights8(g, E * N, K)
            st["w"], st["sw"] = st["w"].view(E, N, K), st["sw"].view(E, N)
        else:
            st["x"] = _rand(g, rows, K).to(torch.bfloat16)
        if op == "experts":
            st["w"] = (_rand(g, E, *((K, N) if kn else (N, K))) * (K ** -0.5)).to(torch.bfloat16)
        if op == "wgrad":
            st["dC"] = (_rand(g, rows, N) * 0.05).to(torch.bfloat16)
            st["dB"] = _rand(g, E, *((K, N) if kn else (N, K))) if case["add"] else torch.zeros((E, K, N) if kn else (E, N, K), device=DEV)
        else:
            st["C"] = torch.zeros((rows, N), device=DEV)
    if own:
        from paper_2401_16677_amd import binding as t3
        st["t3"] = t3
        if "sw" in st:
            st["q"] = torch.empty(st["x"].shape, dtype=torch.int8, device=DEV)
            st["s"] = torch.empty(st["x"].shape[0], device=DEV)
        if op == "linear8":
            st["p"] = t3.problem(M, N, K, 1, 0)
        elif op == "ring8":
            flags = ((t3.T3_FLAG_FWD_DIRECT if case["direct"] else 0) | (t3.T3_FLAG_FWD_BF16 if bf16 else 0)
                     | (t3.T3_FLAG_STEP0_STORE_ONLY if case["step0_store"] else 0))
            st["p"] = t3.problem(M, N, K, tp, case["rank"], case["tile_m"], case["tile_n"], flags=flags)
            t3.t3_track_reset(tp, st["track"])
        else:
            st["p"] = t3.grouped(rows, E, N, K, b_layout=t3.T3_B_KN if kn else t3.T3_B_NK,
                                 flags=t3.T3_GROUPED_ACCUMULATE if case["add"] else 0)
    elif op == "ring8":
        tp = case["tp"]
        for bank in (0, 3 * tp + 2):
            st["track"][bank + 2 * tp:bank + 3 * tp] = -1
        st["gen"] = 0
    return st


# ------------------------------------------------------------------ one pass

def _quantise(x):
    """Each row's largest magnitude is 127; the integer nearest to each quotient, ties to even (quotients in 64 bits: some lie
    next to the border between two integers)."""
    x = x.float()
    top = x.abs().amax(dim=1, keepdim=True)
    q = torch.round(x.double() * 127.0 / torch.where(top > 0, top, torch.ones_like(top)).double()).float()
    return q, top / 127.0


def _plain(st):
    op, case = st["op"], st["case"]
    if op == "linear8":
        q, s = _quantise(st["x"])
        st["C"].copy_(q @ st["w"].float().t() * s * st["sw"])
        return st["C"]
    if op == "ring8":
        M, N, tp, rank = case["M"], case["N"], case["tp"], case["rank"]
        W, R, fwd, t = N // tp, st["R"], st["fwd"], st["track"]
        q, s = _quantise(st["x"])
        C = q @ st["w"].float().t() * s * st["sw"]
        for i in range(tp):
            c = (rank + i) % tp
            cols = slice(c * W, (c + 1) * W)
            total = C[:, cols] if case["step0_store"] and i == 0 else R[:, cols] + C[:, cols]
            if i < tp - 1:
                fwd[i] = total
            if i == tp - 1 or not case["direct"]:
                R[:, cols] = total
        at, other = [(3 * tp + 2) * b for b in (st["gen"] & 1, 1 - (st["gen"] & 1))]
        t[at:at + tp] = -(-M // case["tile_m"]) * -(-W // case["tile_n"])
        t[at + tp:at + 2 * tp] = 1
        t[other:other + 2 * tp] = 0
        st["gen"] += 1
        t[2 * (3 * tp + 2)] = st["gen"]
        return _ring_outputs(st)
    kn, start = case["layout"] == "kn", 0
    q, s = _quantise(st["x"]) if op == "experts8" else (None, None)
    for e, n in enumerate(st["counts"]):
        r = slice(start, start + n)
        start += n
        if op == "experts":
            w = st["w"][e].float()
            st["C"][r] = st["x"][r].float() @ (w if kn else w.t())
        elif op == "experts8":
            st["C"][r] = q[r] @ st["w"][e].float().t() * s[r] * st["sw"][e]
        else:
            x, d = st["x"][r].float(), st["dC"][r].float()
            dB = x.t() @ d if kn else d.t() @ x
            st["dB"][e] = st["dB"][e] + dB if case["add"] else dB
    return st["dB"] if op == "wgrad" else st["C"]


def _ring_outputs(st):
    """The partials, the slots, and what the tracker reports: counters and ready flags of its banks, generation and error (the
    order in which chunks were queued is the device's own)."""
    tp, t = st["case"]["tp"], st["track"]
    bank = 3 * tp + 2
    return [st["R"], st["fwd"], t[:2 * tp], t[bank:bank + 2 * tp], t[2 * bank:2 * bank + 2]]


def run(st):
    if not own:
        return _plain(st)
    op, t3 = st["op"], st["t3"]
    if "q" in st:
        t3.t3_quant_rows(st["x"].shape[0], st["x"].shape[1], st["x"], st["q"], st["s"])
    if op == "linear8":
        t3.t3_gemm_i8(st["p"], st["q"], st["s"], st["w"], st["sw"], st["C"])
        return st["C"]
    if op == "ring8":
        t3.t3_gemm_rs_fused_i8(st["p"], st["q"], st["s"], st["w"], st["sw"], st["R"], st["fwd"], st["track"])
        return _ring_outputs(st)
    if op == "experts":
        t3.t3_gemm_grouped(st["p"], st["offsets"], st["x"], st["w"], st["C"])
        return st["C"]
    if op == "experts8":
        t3.t3_gemm_grouped_i8(st["p"], st["offsets"], st["q"], st["s"], st["w"], st["sw"], st["C"])
        return st["C"]
    t3.t3_gemm_grouped_wgrad(st["p"], st["offsets"], st["x"], st["dC"], st["dB"])
    return st["dB"]


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    op, N, K = case["op"], case["N"], case["K"]
    if op in ("linear8", "ring8"):
        M = case["M"]
        b = 2 * M * K + N * K + 4 * N
        if op == "linear8":
            b += 4 * M * N
        else:
            W, out = N // case["tp"], 2 if case["fwd"] == "bf16" else 4
            b += 4 * M * (N - W if case["step0_store"] else N) + 4 * M * W + out * M * (N - W)
            if not case["direct"]:
                b += 4 * M * (N - W)                    # the sums of forwarded chunks stay in R too
        return {"bytes": b, "flops": 2.0 * M * N * K}
    rows, E = case["rows"], case["groups"]
    used = E * (1.0 - (1.0 - 1.0 / E) ** rows)          # experts that get a row, where all are as likely
    if op == "wgrad":
        b = 2 * rows * (N + K) + 4 * (2 if case["add"] else 1) * E * N * K
    else:
        size = 1 if op == "experts8" else 2
        b = 2 * rows * K + used * N * K * size + 4 * rows * N
    return {"bytes": int(b), "flops": 2.0 * rows * N * K}


# ------------------------------------------------------------------ the definition in 64 bits

def _of_row(x):
    """8-bit values and unit of every row of x, in 64 bits."""
    x = x.double()
    unit = x.abs().max(dim=1).values / 127.0
    q = (x * 127.0 / (x.abs().max(dim=1).values[:, None])).nan_to_num(0.0)
    floor = torch.floor(q)
    up = (q - floor > 0.5) | ((q - floor == 0.5) & (torch.remainder(floor, 2.0) == 1.0))
    return floor + up.double(), unit


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op in ("linear8", "ring8"):
        q, unit = _of_row(st["x"])
        C = torch.mm(q, st["w"].double().t()) * torch.outer(unit, st["sw"].double())
        if op == "linear8":
            return C
        tp, rank, W = case["tp"], case["rank"], case["N"] // case["tp"]
        total = st["R"].double() + C
        if case["step0_store"]:
            total[:, rank * W:(rank + 1) * W] = C[:, rank * W:(rank + 1) * W]
        order = [(rank + i) % tp for i in range(tp - 1)]
        fwd = torch.stack([total[:, c * W:(c + 1) * W] for c in order])
        R = st["R"].double()
        for c in range(tp):
            if c not in order or not case["direct"]:
                R[:, c * W:(c + 1) * W] = total[:, c * W:(c + 1) * W]
        return [R, fwd, None, None, None]
    ends = torch.tensor(st["counts"]).cumsum(0).tolist()
    spans = list(zip([0] + ends[:-1], ends))
    if op == "wgrad":
        pair = (st["x"], st["dC"]) if case["layout"] == "kn" else (st["dC"], st["x"])
        grad = torch.stack([torch.mm(pair[0][a:b].double().t(), pair[1][a:b].double()) for a, b in spans])
        return grad + st["dB"].double()
    C = torch.zeros(st["C"].shape, dtype=torch.float64, device=DEV)
    q, unit = _of_row(st["x"]) if op == "experts8" else (st["x"].double(), None)
    for e, (a, b) in enumerate(spans):
        w = st["w"][e].double()
        C[a:b] = torch.mm(q[a:b], w if case["layout"] == "kn" else w.t())
        if op == "experts8":
            C[a:b] *= torch.outer(unit[a:b], st["sw"][e].double())
    return C
