"""The operators of a block-pruned feed-forward layer of a language model, as a serving program calls them: the root mean
square norm with the residual's addition and 8-bit rows, rows to 8 bits, and the product with a block-pruned weight (plain
and gated) with bias, activation and residual in its epilogue.

Sizes are generic layer widths; sparsities and block lengths are those of this repository's own sweep (50 ... 90 %, blocks of
2, 4, 8, 16 output rows at one input channel, starting at any row)."""
import math

import torch

own = False   # True: run() calls the library's operators; False: their plain form in 32 bits

BF16, F16, E4M3 = "bf16", "f16", "e4m3"
TYPES = {BF16: torch.bfloat16, F16: torch.float16, E4M3: torch.float8_e4m3fn, "f32": torch.float32}
SIZE = {BF16: 2, F16: 2, E4M3: 1, "f32": 4}
E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -126
EPS = 1e-5


# ------------------------------------------------------------------ cases
def listed():
    def norm(name, T, C, dt, pad=0):
        return {"name": name, "op": "norm", "T": T, "C": C, "dtype": dt, "pad": pad}

    def rows(name, T, C, dt, pad=0):
        return {"name": name, "op": "rows", "T": T, "C": C, "dtype": dt, "pad": pad}

    def product(name, T, M, C, dt, out, Nb, p, act, gated=False, residual=False, bias=False, pad=0):
        return {"name": name, "op": "product", "T": T, "M": M, "C": C, "dtype": dt, "out": out, "Nb": Nb, "p": p, "act": act,
                "gated": gated, "residual": residual, "bias": bias, "pad": pad}

    return [
        # one token of a running answer enters a layer: latency only
        norm("norm_token", 1, 4096, BF16),
        # a batch of prompts of uneven length, an odd width, rows cut out of a wider buffer (nothing 16-byte aligned)
        norm("norm_ragged", 1531, 2051, F16, pad=3),
        # long prompts of a wide model: bandwidth
        norm("norm_prompt", 16384, 8192, BF16),
        # hidden activations of three running answers go to 8 bits in front of the second product
        rows("rows_batch", 3, 16384, BF16),
        # the same for long prompts
        rows("rows_prompt", 8192, 16384, BF16),
        # one token through an output projection, 80 % pruned: the kept weights are all there is to read
        product("product_token", 1, 4096, 4096, BF16, BF16, 4, 80, "none", residual=True),
        # a batch of 24 running answers through the second product of a feed-forward layer
        product("product_batch", 24, 4096, 8192, F16, F16, 8, 70, "none", residual=True, bias=True),
        # a small model with odd sizes: rows not 16-byte aligned, biased GELU layer
        product("product_ragged", 777, 1500, 1003, BF16, BF16, 2, 70, "gelu", bias=True, pad=4),
        # long prompts through the second product: dense rate
        product("product_prompt", 8192, 4096, 8192, BF16, BF16, 4, 50, "none", residual=True),
        # one token through gate and up projections in 8 bits
        product("gated_token", 1, 16384, 4096, E4M3, BF16, 4, 80, "silu", gated=True),
        # 64 running answers, gated GELU
        product("gated_batch", 64, 8192, 2048, BF16, BF16, 4, 70, "gelu_tanh", gated=True),
        # long prompts through gate and up projections in 8 bits
        product("gated_prompt", 8192, 16384, 4096, E4M3, BF16, 4, 50, "silu", gated=True),
    ]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(["norm", "rows", "product", "product", "product"])
    pad = rng.choice([0, 0, 8, 1, 5])
    if op != "product":
        C = _log(rng, 64, 16384)
        if rng.random() < 0.5:
            C = max(64, C // 64 * 64)
        T = _log(rng, 1, min(16384, (1 << 27) // C))
        return {"op": op, "T": T, "C": C, "dtype": rng.choice([BF16, F16]), "pad": pad}
    T = _log(rng, 1, 8192)
    gated = rng.random() < 0.4
    C = _log(rng, 128, 8192)
    M = _log(rng, 128, 8192)
    if rng.random() < 0.5:
        C, M = max(128, C // 128 * 128), max(128, M // 128 * 128)
    if gated:
        M -= M % 2
    if 3072 in (C, M):
        C, M = C + 128 * (C == 3072), M + 128 * (M == 3072)
    dt = rng.choice([BF16, F16, E4M3])
    return {"op": op, "T": T, "M": M, "C": C, "dtype": dt, "out": rng.choice([BF16, F16]) if dt == E4M3 else dt,
            "Nb": rng.choice([2, 4, 8, 16]), "p": rng.choice([50, 70, 80, 90]),
            "act": rng.choice(["silu", "gelu", "gelu_tanh", "relu"] if gated else ["none", "none", "relu", "gelu", "silu"]),
            "gated": gated, "residual": rng.random() < 0.5, "bias": rng.random() < 0.5, "pad": pad}


# ------------------------------------------------------------------ inputs
def _rand(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _rows_of(values, dtype, pad):
    """The values as rows of a buffer `pad` elements wider: what a slice of a larger activation looks like."""
    T, C = values.shape
    buf = torch.zeros(T, C + pad, dtype=dtype, device="cuda")
    buf[:, :C] = values.to(dtype)
    return buf[:, :C]


def _activations(g, T, C):
    """Hidden states: unit variance, a few strong channels, tokens of different size."""
    strong = torch.where(torch.rand(C, generator=g, device="cuda") < 0.01, 8.0, 1.0)
    return _rand(g, T, C) * strong * torch.exp(0.3 * _rand(g, T, 1))


def _weight(g, case):
    """A pruned weight: c blocks of Nb rows in each input channel at uniform non-overlapping places. Returns the weight
    with zeros where pruned (fp32) and the mask."""
    M, C, Nb = case["M"], case["C"], case["Nb"]
    c = max(1, M * (100 - case["p"]) // (100 * Nb))
    free = M - c * (Nb - 1)
    at = torch.rand(C, free, generator=g, device="cuda").argsort(1)[:, :c].sort(1).values
    start = at + torch.arange(c, device="cuda") * (Nb - 1)
    kept = (start[:, :, None] + torch.arange(Nb, device="cuda")).reshape(C, c * Nb)
    mask = torch.zeros(C, M, dtype=torch.uint8, device="cuda").scatter_(1, kept, 1).t().contiguous()
    return _rand(g, M, C) * (1.0 / math.sqrt(C * (100 - case["p"]) / 100)) * mask, mask


def _quantised(v):
    """Rows in 8 bits and their scales."""
    s = (v.abs().amax(1, keepdim=True) / E4M3_MAX).clamp_min(SCALE_MIN)
    return (v / s).to(torch.float8_e4m3fn), s[:, 0].contiguous()


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    T, C, dt, pad = case["T"], case["C"], case["dtype"], case["pad"]
    d = {}
    if case["op"] == "norm":
        d["x"] = _rows_of(0.5 * _activations(g, T, C), TYPES[dt], pad)
        d["residual"] = _rows_of(_activations(g, T, C), TYPES[dt], pad)
        d["gamma"] = (1.0 + 0.2 * _rand(g, C)).to(TYPES[dt])
    elif case["op"] == "rows":
        d["x"] = _rows_of(_activations(g, T, C), TYPES[dt], pad)
    else:
        M = case["M"]
        F = M // 2 if case["gated"] else M
        d["W"], d["mask"] = _weight(g, case)
        a = _activations(g, T, C)
        if dt == E4M3:
            q, d["x_scales"] = _quantised(a)
            d["x"] = _rows_of(q.float(), TYPES[dt], pad)
            d["w"], d["w_scales"] = _quantised(d["W"])
        else:
            d["x"], d["x_scales"] = _rows_of(a, TYPES[dt], pad), None
            d["w"], d["w_scales"] = d["W"].to(TYPES[dt]), None
        d["bias"] = 0.1 * _rand(g, M) if case["bias"] else None
        d["residual"] = _rows_of(_rand(g, T, F), TYPES[case["out"]], 0) if case["residual"] else None
    return d


def prepare(case, seed):
    d = _inputs(case, seed)
    state = {"case": case, "in": d}
    if case["op"] == "product":
        W, mask = d.pop("W"), d.pop("mask")
        if own:   # a program keeps the packed layer on the device, not the dense weight
            import paper_2407_19644_b200 as ubp
            del d["w"], d["w_scales"]
            blob = ubp.ubp_pack(W.cpu().numpy(), mask.cpu().numpy(), case["Nb"])
            state["plan"] = ubp.LinearPlan(blob, dtype=TYPES[case["dtype"]], gated=case["gated"])
    return state


# ------------------------------------------------------------------ one pass
def _act(v, act):
    if act == "relu":
        return v.clamp_min(0.0)
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _run_own(state):
    import paper_2407_19644_b200 as ubp
    case, d = state["case"], state["in"]
    if case["op"] == "norm":
        q, s, h = ubp.ubp_rmsnorm(d["x"], d["gamma"], EPS, residual=d["residual"], out_dtype=torch.float8_e4m3fn)
        return {"q": q, "scales": s, "h": h}
    if case["op"] == "rows":
        q, s = ubp.ubp_quant_rows(d["x"])
        return {"q": q, "scales": s}
    return {"y": ubp.ubp_linear(state["plan"], d["x"], bias=d["bias"], activation=case["act"], residual=d["residual"],
                                x_scales=d["x_scales"], out_dtype=TYPES[case["out"]])}


def run(state):
    if own:
        return _run_own(state)
    case, d = state["case"], state["in"]
    if case["op"] == "norm":
        h = d["x"].float() + d["residual"].float()
        y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * d["gamma"].float()
        q, s = _quantised(y)
        return {"q": q, "scales": s, "h": h.to(TYPES[case["dtype"]])}
    if case["op"] == "rows":
        q, s = _quantised(d["x"].float())
        return {"q": q, "scales": s}
    z = d["x"].float() @ d["w"].float().t()
    if d["x_scales"] is not None:
        z = z * d["x_scales"][:, None] * d["w_scales"][None, :]
    if d["bias"] is not None:
        z = z + d["bias"]
    if case["gated"]:
        F = case["M"] // 2
        y = _act(z[:, :F], case["act"]) * z[:, F:]
    else:
        y = _act(z, case["act"])
    if d["residual"] is not None:
        y = y + d["residual"].float()
    return {"y": y.to(TYPES[case["out"]])}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    T, C = case["T"], case["C"]
    n = T * C
    if case["op"] == "norm":      # x and residual in, h and 8-bit rows out; add, square, sum, two products, maximum, division
        b = SIZE[case["dtype"]]
        return {"bytes": n * (3 * b + 1) + C * b + 4 * T, "flops": 7.0 * n}
    if case["op"] == "rows":
        return {"bytes": n * (SIZE[case["dtype"]] + 1) + 4 * T, "flops": 2.0 * n}
    M, Nb = case["M"], case["Nb"]
    F = M // 2 if case["gated"] else M
    blocks = C * max(1, M * (100 - case["p"]) // (100 * Nb))
    b, o = SIZE[case["dtype"]], SIZE[case["out"]]
    # activations, kept weights with one 16-bit channel index a block, outputs; multiply-adds of kept weights only
    nbytes = n * b + blocks * (Nb * b + 2) + T * F * o * (2 if case["residual"] else 1) + (4 * M if case["bias"] else 0)
    if case["dtype"] == E4M3:
        nbytes += 4 * (T + M)
    return {"bytes": nbytes, "flops": 2.0 * blocks * Nb * T}


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    d = _inputs(case, seed)
    if case["op"] == "rows":
        x = d["x"].double()
        s = torch.clamp(torch.linalg.vector_norm(x, ord=math.inf, dim=1) / E4M3_MAX, min=SCALE_MIN)
        return {"q": x / s.unsqueeze(1), "scales": s}
    if case["op"] == "norm":
        h = torch.add(d["x"].double(), d["residual"].double())
        rms = torch.sqrt(torch.linalg.vector_norm(h, dim=1).square() / case["C"] + EPS)
        y = h / rms.unsqueeze(1) * d["gamma"].double()
        s = torch.clamp(torch.linalg.vector_norm(y, ord=math.inf, dim=1) / E4M3_MAX, min=SCALE_MIN)
        return {"q": y / s.unsqueeze(1), "scales": s, "h": h}
    x, w = d["x"].double(), d["w"].double()
    if case["dtype"] == E4M3:
        x, w = x * d["x_scales"].double().unsqueeze(1), w * d["w_scales"].double().unsqueeze(1)
    z = torch.einsum("tc,mc->tm", x, w)
    if case["bias"]:
        z += d["bias"].double()
    z, up = z.chunk(2, dim=1) if case["gated"] else (z, None)
    act = {"none": lambda v: v, "relu": torch.relu, "silu": lambda v: v * torch.sigmoid(v),
           "gelu": torch.nn.functional.gelu, "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[case["act"]]
    y = act(z) if up is None else act(z) * up
    if case["residual"]:
        y = y + d["residual"].double()
    return {"y": y}
