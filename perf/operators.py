"""The operators of a transformer's feed-forward part in FP8, as cases that can be timed and compared.

  linear        product of FP8 operands with bias, activation and residual in its epilogue; the value before
                the activation kept for the backward pass (fp8_gemm_act)
  linear_grad   data gradient through the next layer's weight, times the activation's derivative, with the
                bias gradient (fp8_gemm_act_grad)
  gated         both projections of a gated feed-forward block, activation and product in one pass
                (fp8_gemm_gated)
  gated_grad    its backward pass: gradient of the block's inner product through the down projection's
                weight, and out of that the gradients of both projections (fp8_gemm_gated_grad)
  clip          global norm of many gradient tensors and their clipping to it (fp8_grad_norm, fp8_grad_clip)

Operands are FP8 bytes with one scaling factor each, as the cast before the product leaves them; weights are stored
[out, in] unless a case says otherwise.  Where `own` is true, run() calls the library; else it computes the same in 32 bits
out of elementary tensor operations.
"""
import math

import torch

own = False

FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
MOST = {"e4m3": 448.0, "e5m2": 57344.0}
WIDER = {"bf16": torch.bfloat16, "f32": torch.float32}
MOST_FLOPS = 1e12          # of a drawn product (the largest listed one takes ten times as many)


def _linear(name, M, N, K, act, out, bias=True, residual=False, z=None, amax=False, weight="out_in", fp8_instructions=False):
    return {"name": name, "kind": "linear", "M": M, "N": N, "K": K, "act": act, "out": out, "bias": bias, "residual": residual,
            "z": z, "amax": amax, "weight": weight, "fp8_instructions": fp8_instructions}


def _linear_grad(name, M, N, K, act, out, z="bf16", dbias=True, amax=False, fp8_instructions=False):
    return {"name": name, "kind": "linear_grad", "M": M, "N": N, "K": K, "act": act, "out": out, "z": z, "dbias": dbias, "amax": amax,
            "fp8_instructions": fp8_instructions}


def _gated(name, M, F, K, act, out, gu=None, amax=False, fp8_instructions=False):
    return {"name": name, "kind": "gated", "M": M, "F": F, "K": K, "act": act, "out": out, "gu": gu, "amax": amax, "fp8_instructions": fp8_instructions}


def _gated_grad(name, M, F, K, act, out, gu="bf16", amax=False, fp8_instructions=False):
    return {"name": name, "kind": "gated_grad", "M": M, "F": F, "K": K, "act": act, "out": out, "gu": gu, "amax": amax, "fp8_instructions": fp8_instructions}


def _clip(name, layers, width, inner, dtype, ragged=0, clips=True):
    return {"name": name, "kind": "clip", "layers": layers, "width": width, "inner": inner, "dtype": dtype, "ragged": ragged, "clips": clips}


def listed():
    return [
        # one token through the up projection of the small-GPT layer while text is generated: the smallest call
        _linear("linear_1_token", 1, 6144, 2048, "gelu_tanh", "bf16"),
        # the same projection in training: FP8 output for the next product with its maximum, pre-activation kept
        _linear("linear_train_fp8_out", 4096, 6144, 2048, "gelu", "e4m3", z="bf16", amax=True),
        # the down projection back onto the residual stream, a ragged batch
        _linear("linear_down_residual", 3001, 2048, 6144, "none", "bf16", residual=True),
        # backward of the up projection: gradient through the down projection's weight, E5M2 output for the next products
        _linear_grad("linear_grad_train", 4096, 6144, 2048, "gelu", "e5m2", amax=True),
        # the same for a short ragged batch and an odd width, everything kept in 32 bits
        _linear_grad("linear_grad_ragged_f32", 777, 1000, 2048, "relu", "f32", z="f32"),
        # one token through the gated block of a small model
        _gated("gated_1_token", 1, 6144, 2048, "silu", "bf16"),
        # sixteen tokens through a block of the 175B-class width: the stream of the weights is all of it
        _gated("gated_16_tokens_175b", 16, 24576, 12288, "silu", "bf16"),
        # that block's forward pass in training on the FP8 matrix instructions: the largest product
        _gated("gated_train_175b_fp8", 8192, 24576, 12288, "silu", "bf16", gu="bf16", fp8_instructions=True),
        # backward of a gated block, gradients of both projections in E5M2 for the two products that follow
        _gated_grad("gated_grad_train", 8192, 6144, 2048, "silu", "e5m2", amax=True),
        # the same for a ragged batch on the FP8 matrix instructions, 16-bit gradients
        _gated_grad("gated_grad_ragged_fp8", 1537, 5504, 4096, "gelu_tanh", "bf16", fp8_instructions=True),
        # all gradients of a model of 24 layers, 16 bits
        _clip("clip_24_layers", 24, 2048, 6144, "bf16"),
        # a few small tensors of odd sizes, 32 bits: launches and latency
        _clip("clip_small_ragged_f32", 2, 130, 257, "f32", ragged=1),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def _width(rng, lo=64, hi=12288):
    """A layer width: mostly a multiple of 64, now and then of 16, now and then anything."""
    v, r = _spread(rng, lo, hi), rng.random()
    if r < 0.75:
        return max(64, (v + 32) // 64 * 64)
    return max(16, (v + 8) // 16 * 16) if r < 0.9 else v


def _sizes(rng, wide=1):
    while True:
        m, n, k = _spread(rng, 1, 8192), _width(rng), _width(rng)
        if 2.0 * m * n * k * wide <= MOST_FLOPS:
            return m, n, k


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear_grad", "gated", "gated", "gated_grad", "clip"])
    if kind == "clip":
        while True:
            c = _clip("", _spread(rng, 1, 48), _spread(rng, 64, 6144), _spread(rng, 64, 12288), rng.choice(["bf16", "f32"]), rng.choice([0, 0, 1]), rng.random() < 0.7)
            if sum(_clip_sizes(c)) <= 1 << 30:
                break
    else:
        act, fast = rng.choice(["relu", "gelu", "gelu_tanh", "silu"]), rng.random() < 0.4
        m, n, k = _sizes(rng, 2 if kind == "gated" else 1)
        out = rng.choice(["bf16", "bf16", "e4m3" if kind in ("linear", "gated") else "e5m2"] + ([] if fast else ["f32"]))
        # (sums of the FP8 instructions are not shown in 32 bits)
        amax, kept = not fast and out in FORMATS, rng.choice([None, "bf16", "bf16"])
        if kind == "linear":
            c = _linear("", m, n, k, rng.choice([act, "none"]), out, rng.random() < 0.7, rng.random() < 0.3, kept, amax, rng.choice(["out_in", "out_in", "in_out"]), fast)
        elif kind == "linear_grad":
            c = _linear_grad("", m, n, k, act, out, rng.choice(["bf16", "bf16", "f32"]), not fast and rng.random() < 0.7, amax, fast)
        elif kind == "gated":
            c = _gated("", m, n, k, act, out, kept, amax, fast)
        else:
            c = _gated_grad("", m, n, k, act, out, rng.choice(["bf16", "bf16", "f32"]), amax, fast)
    del c["name"]
    return c


def _clip_sizes(case):
    """Elements of the gradient tensors: per layer four weights, two biases, two norm weights; then a final norm."""
    w, f, odd = case["width"], case["inner"], case["ragged"]
    layer = [3 * w * w + odd, w * w, f * w, f, w * f + odd, w, w, w]
    return layer * case["layers"] + [w]


# ---- inputs --------------------------------------------------------------------------------------------------------------
def _bytes(x, fmt):
    """(FP8 bytes, factor): per-tensor scaling, the largest magnitude at the format's largest value."""
    scale = (MOST[fmt] / x.abs().amax().float()).reshape(1)
    return (x * scale).clamp(-MOST[fmt], MOST[fmt]).to(FORMATS[fmt]).view(torch.uint8), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device="cuda").mul_(std)

    kind = case["kind"]
    s = {"case": case}
    if kind == "clip":
        sizes, dtype = _clip_sizes(case), WIDER[case["dtype"]]
        total = sum(sizes)
        std = 1e-3
        flat = torch.empty(total, dtype=dtype, device="cuda")
        for i in range(0, total, 1 << 26):
            flat[i:i + (1 << 26)] = normal(min(1 << 26, total - i), std=std)
        s["flat"], s["out"] = flat, torch.empty_like(flat)
        s["xs"], s["outs"] = list(flat.split(sizes)), list(s["out"].split(sizes))
        s["max_norm"] = std * math.sqrt(total) * (0.3 if case["clips"] else 4.0)
        s["norm"] = torch.zeros(1, device="cuda")
        s["workspace"] = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
        return s
    M, K = case["M"], case["K"]
    N = case["N"] if "N" in case else case["F"]
    grad = kind in ("linear_grad", "gated_grad")
    # activations with a few channels that stick out; gradients are small and in E5M2
    x = normal(M, K, std=1e-5 if grad else 1.0)
    if not grad:
        x[:, :: max(1, K // 4)] *= 10.0
    s["A"], s["sA"] = _bytes(x, "e5m2" if grad else "e4m3")
    del x
    rows = 2 * N if kind == "gated" else N
    w = normal(rows, K, std=K ** -0.5)
    s["B"], s["sB"] = _bytes(w, "e4m3")
    del w
    # the weight of a data gradient lies [in of this product, out of it]; the others [out, in] or as the case says
    if grad or case.get("weight") == "in_out":
        s["B"] = s["B"].t().contiguous()
    wide = 2 * N if kind == "gated_grad" else N
    out = case["out"]
    s["D"] = torch.empty((M, wide), dtype=WIDER.get(out, torch.uint8), device="cuda")
    # a factor from past maxima: outputs of the size that these inputs give fit the format (a rare one saturates)
    s["sD"] = torch.full((1,), MOST[out] / (4e-5 if grad else 24.0), device="cuda") if out in FORMATS else None
    s["amax"] = torch.zeros(1, device="cuda") if case["amax"] else None
    if kind == "linear":
        s["bias"] = normal(N, std=0.1).to(torch.bfloat16) if case["bias"] else None
        s["residual"] = normal(M, N).to(torch.bfloat16) if case["residual"] else None
        s["Z"] = torch.empty((M, N), dtype=WIDER[case["z"]], device="cuda") if case["z"] else None
    elif kind == "linear_grad":
        s["Z"] = normal(M, N).to(WIDER[case["z"]])
        s["dbias"] = torch.empty(N, device="cuda") if case["dbias"] else None
        # (a row of partial sums for every 32 rows of the output)
        s["workspace"] = torch.empty(((M + 31) // 32) * 4 * N, dtype=torch.uint8, device="cuda") if case["dbias"] else None
    elif kind == "gated":
        s["GU"] = torch.empty((M, 2 * N), dtype=WIDER[case["gu"]], device="cuda") if case["gu"] else None
    else:
        s["GU"] = normal(M, 2 * N).to(WIDER[case["gu"]])
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------
def _result(case, s, **more):
    d = s["D"].view(FORMATS[case["out"]]) if case["out"] in FORMATS else s["D"]
    return {k: v for k, v in dict(out=d, amax=s["amax"], **more).items() if v is not None}


def _run_own(s):
    import paper_2209_05433_amd as fp8
    case = s["case"]
    kind = case["kind"]
    if kind == "clip":
        fp8.fp8_grad_norm(s["xs"], s["norm"], s["workspace"])
        fp8.fp8_grad_clip(s["xs"], s["norm"], s["max_norm"], s["outs"])
        return {"out": s["out"], "norm": s["norm"]}
    act = {"none": fp8.FP8_ACT_NONE, "relu": fp8.FP8_ACT_RELU, "gelu": fp8.FP8_ACT_GELU, "gelu_tanh": fp8.FP8_ACT_GELU_TANH, "silu": fp8.FP8_ACT_SILU}[case["act"]]
    out = {"f32": fp8.FP8_OUT_F32, "bf16": fp8.FP8_OUT_BF16, "e4m3": fp8.FP8_OUT_E4M3, "e5m2": fp8.FP8_OUT_E5M2}[case["out"]]
    flags = fp8.FP8_GEMM_MFMA8 if case["fp8_instructions"] else 0
    E4M3, E5M2 = fp8.FP8_E4M3, fp8.FP8_E5M2
    if kind == "linear":
        fp8.fp8_gemm_act(s["A"], E4M3, False, s["B"], E4M3, case["weight"] == "out_in", s["D"], out, s["sA"], s["sB"], act,
                         s["bias"], s["residual"], s["Z"], s["sD"], s["amax"], flags)
        return _result(case, s, z=s["Z"])
    if kind == "linear_grad":
        fp8.fp8_gemm_act_grad(s["A"], E5M2, False, s["B"], E4M3, False, s["D"], out, s["sA"], s["sB"], act, s["Z"],
                              s["dbias"], s["workspace"], s["sD"], s["amax"], flags)
        return _result(case, s, dbias=s["dbias"])
    if kind == "gated":
        fp8.fp8_gemm_gated(s["A"], E4M3, False, s["B"], E4M3, True, s["D"], out, s["sA"], s["sB"], act, s["GU"], s["sD"], s["amax"], flags)
        return _result(case, s, gu=s["GU"])
    fp8.fp8_gemm_gated_grad(s["A"], E5M2, False, s["B"], E4M3, False, s["D"], out, s["sA"], s["sB"], act, s["GU"], s["sD"], s["amax"], flags)
    return _result(case, s)


def _act(z, act):
    if act == "none":
        return z
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))


def _act_grad(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z * z * z))
    return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)


def _out(y, s, case):
    out = case["out"]
    if out in WIDER:
        return y.to(WIDER[out])
    return (y * s["sD"]).clamp(-MOST[out], MOST[out]).to(FORMATS[out])


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "clip":
        x = s["flat"].float()
        norm = x.square().sum().sqrt().reshape(1)
        coefficient = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
        return {"out": (x * coefficient).to(s["flat"].dtype), "norm": norm}
    grad = kind in ("linear_grad", "gated_grad")
    a = s["A"].view(FORMATS["e5m2" if grad else "e4m3"]).float()
    b = s["B"].view(FORMATS["e4m3"]).float()
    y = torch.matmul(a, b if grad or case.get("weight") == "in_out" else b.t())
    y = y / (s["sA"] * s["sB"])
    more = {}
    if kind == "linear":
        z = y if s["bias"] is None else y + s["bias"].float()
        if case["z"]:
            more["z"] = z.to(WIDER[case["z"]])
        y = _act(z, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
    elif kind == "linear_grad":
        y = y * _act_grad(s["Z"].float(), case["act"])
        if case["dbias"]:
            more["dbias"] = y.sum(0)
    elif kind == "gated":
        if case["gu"]:
            more["gu"] = y.to(WIDER[case["gu"]])
        g, u = y.chunk(2, dim=1)
        y = _act(g, case["act"]) * u
    else:
        g, u = s["GU"].float().chunk(2, dim=1)
        y = torch.cat([y * u * _act_grad(g, case["act"]), y * _act(g, case["act"])], dim=1)
    if case["amax"]:
        more["amax"] = y.abs().amax().reshape(1)
    return {"out": _out(y, s, case), **more}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- in 64 bits -------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "clip":
        x = s["flat"].double()
        norm = torch.linalg.vector_norm(x)
        return {"out": x.mul_(min(1.0, s["max_norm"] / (float(norm) + 1e-6))), "norm": norm.reshape(1)}
    grad = kind in ("linear_grad", "gated_grad")
    a = s["A"].view(FORMATS["e5m2" if grad else "e4m3"]).double()
    b = s["B"].view(FORMATS["e4m3"]).double()
    if not (grad or case.get("weight") == "in_out"):
        b = b.t()
    y = (a @ b).div_(float(s["sA"]) * float(s["sB"]))
    del a, b

    sigmoid = torch.sigmoid

    def value(t):
        name = case["act"]
        if name == "gelu":
            return t * torch.special.ndtr(t)
        if name == "gelu_tanh":
            return t * sigmoid(2 * math.sqrt(2 / math.pi) * (t + 0.044715 * t ** 3))
        return {"none": lambda: t, "relu": lambda: torch.relu(t), "silu": lambda: t * sigmoid(t)}[name]()

    def slope(t):
        t = t.detach().requires_grad_(True)
        with torch.enable_grad():
            return torch.autograd.grad(value(t).sum(), t)[0]

    res = {}
    if kind == "linear":
        z = y if s["bias"] is None else y + s["bias"].double()
        if case["z"]:
            res["z"] = z
        y = value(z) if s["residual"] is None else value(z) + s["residual"].double()
    elif kind == "linear_grad":
        y = y * slope(s["Z"].double())
        if case["dbias"]:
            res["dbias"] = y.sum(0)
    elif kind == "gated":
        if case["gu"]:
            res["gu"] = y
        y = value(y[:, :case["F"]]) * y[:, case["F"]:]
    else:
        gu = s["GU"].double()
        g, u = gu[:, :case["F"]], gu[:, case["F"]:]
        y = torch.cat([y * u * slope(g), y * value(g)], 1)
    if case["amax"]:
        res["amax"] = y.abs().max().reshape(1)
    if case["out"] in FORMATS:
        y = (y * float(s["sD"])).clamp(-MOST[case["out"]], MOST[case["out"]])
    return {"out": y, **res}


def work(case):
    kind = case["kind"]
    if kind == "clip":
        n, size = sum(_clip_sizes(case)), 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 2 * n * size + 4, "flops": 3 * n}
    M, K = case["M"], case["K"]
    N = case["N"] if "N" in case else case["F"]
    size = {"bf16": 2, "f32": 4, "e4m3": 1, "e5m2": 1, None: 0}
    columns = 2 * N if kind == "gated" else N
    moved = M * K + columns * K + M * (2 * N if kind == "gated_grad" else N) * size[case["out"]]
    if kind == "linear":
        moved += M * N * size[case["z"]] + (2 * N if case["bias"] else 0) + (2 * M * N if case["residual"] else 0)
    elif kind == "linear_grad":
        moved += M * N * size[case["z"]] + (4 * N if case["dbias"] else 0)
    else:
        moved += M * 2 * N * size[case["gu"]]
    return {"bytes": moved, "flops": 2 * M * columns * K}
