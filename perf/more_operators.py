"""The two ends of a training step around the products, as cases that can be timed and compared.

  loss        softmax cross entropy of the logits x w^T over a vocabulary, in the product's epilogue: no logits in memory
              (fp8_gemm_xent)
  loss_grad   the logits' gradient for the two products that follow, out of a second product and the kept
              logarithms of the sums (fp8_gemm_xent_grad)
  adamw       AdamW over all tensors of a model, clipping and the weights' FP8 copies in the same pass, with
              states in 32 bits or in FP8 with a factor for each 128 of them (fp8_adamw)

Products take FP8 bytes with one scaling factor an operand; weights are stored [out, in] unless a case says otherwise.  Where
`own` is true, run() calls the library; else it computes the same in 32 bits out of elementary tensor operations.
"""
import math

import torch

own = False

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
WIDER = {"bf16": torch.bfloat16, "f32": torch.float32}
VOCABULARY = 50257
MOST_FLOPS = 1e12          # of a drawn product (the largest listed one takes ten times as many)
BLOCK = 128                # state elements that share a factor


def _loss(name, M, N, K, z_weight=0.0, first=0, weight="out_in"):
    return {"name": name, "kind": "loss", "M": M, "N": N, "K": K, "z_weight": z_weight, "first": first, "weight": weight}


def _loss_grad(name, M, N, K, out, z_weight=0.0, first=0, weight="out_in", each_row=False, amax=False, fp8_instructions=False):
    return {"name": name, "kind": "loss_grad", "M": M, "N": N, "K": K, "out": out, "z_weight": z_weight, "first": first, "weight": weight,
            "each_row": each_row, "amax": amax, "fp8_instructions": fp8_instructions}


def _adamw(name, layers, width, inner, state, param="f32", grad="bf16", copies=True, clips=True, ragged=0):
    return {"name": name, "kind": "adamw", "layers": layers, "width": width, "inner": inner, "state": state, "param": param, "grad": grad,
            "copies": copies, "clips": clips, "ragged": ragged}


def listed():
    return [
        # how likely one token of a small model is: the stream of the weight
        _loss("loss_1_token", 1, VOCABULARY, 2048),
        # a training batch of the small model, with the term that keeps the sums near 1
        _loss("loss_small_gpt", 4096, VOCABULARY, 2048, z_weight=1e-4),
        # the second of eight pieces of a vocabulary that is split over GPUs: most labels lie in other pieces
        _loss("loss_ragged_piece", 1001, 6283, 4096, first=6283),
        # a training batch of the 175B-class width: the largest forward product
        _loss("loss_175b", 8192, VOCABULARY, 12288),
        # gradient of a short sequence
        _loss_grad("loss_grad_64_tokens", 64, VOCABULARY, 2048, "e5m2", amax=True),
        # the small model's batch: E5M2 for the two products that follow, with the maximum for the next step's factor
        _loss_grad("loss_grad_small_gpt", 4096, VOCABULARY, 2048, "e5m2", z_weight=1e-4, amax=True),
        # a ragged batch, rows weighted one by one, 16-bit gradient
        _loss_grad("loss_grad_ragged_bf16", 777, 30011, 4096, "bf16", z_weight=1e-4, each_row=True),
        # the 175B-class batch on the FP8 matrix instructions
        _loss_grad("loss_grad_175b_fp8", 8192, VOCABULARY, 12288, "e5m2", fp8_instructions=True),
        # all tensors of a model of 24 layers, master weights and states in 32 bits, clipped, weights left in FP8 for the next step
        _adamw("adamw_24_layers_f32", 24, 2048, 6144, "f32"),
        # the same with states in 8 bits
        _adamw("adamw_24_layers_fp8", 24, 2048, 6144, "fp8"),
        # a few small tensors of odd sizes: launches and latency
        _adamw("adamw_small_f32", 2, 130, 257, "f32", grad="f32", copies=False, ragged=1),
        # the same with states in 8 bits and 16-bit weights
        _adamw("adamw_small_fp8", 2, 130, 257, "fp8", param="bf16", copies=False, clips=False, ragged=1),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["loss", "loss", "loss_grad", "loss_grad", "adamw", "adamw"])
    if kind == "adamw":
        while True:
            c = _adamw("", _spread(rng, 1, 24), _spread(rng, 64, 4096), _spread(rng, 64, 8192), rng.choice(["f32", "fp8"]), rng.choice(["f32", "f32", "bf16"]),
                       rng.choice(["bf16", "f32"]), rng.random() < 0.6, rng.random() < 0.7, rng.choice([0, 0, 1, 3]))
            if sum(_sizes(c)) <= 1 << 29:
                break
    else:
        while True:
            m, n = _spread(rng, 1, 16384), _spread(rng, 1000, 200000)
            k, r = _spread(rng, 64, 12288), rng.random()
            k = max(64, (k + 32) // 64 * 64) if r < 0.7 else max(16, (k + 8) // 16 * 16) if r < 0.9 else k
            if 2.0 * m * n * k <= MOST_FLOPS and m * n <= 1 << 29:
                break
        z, first = rng.choice([0.0, 1e-4]), rng.choice([0, 0, 0, n])
        # (weights [in, out] mostly of padded vocabularies)
        weight = rng.choice(["out_in", "out_in", "out_in", "in_out"])
        if weight == "in_out" and rng.random() < 0.7:
            n = (n + 63) // 64 * 64
        if kind == "loss":
            c = _loss("", m, n, k, z, first, weight)
        else:
            fast, out = rng.random() < 0.4, rng.choice(["e5m2", "e5m2", "bf16", "f32"])
            # (sums of the FP8 instructions are not shown in 32 bits)
            fast = fast and out != "f32"
            c = _loss_grad("", m, n, k, out, z, first, weight, rng.random() < 0.3, not fast and out == "e5m2", fast)
    del c["name"]
    return c


def _sizes(case):
    """Elements of the tensors: per layer four weights, two biases, two norm weights; then a final norm."""
    w, f, odd = case["width"], case["inner"], case["ragged"]
    layer = [3 * w * w + odd, w * w, f * w, f, w * f + odd, w, w, w]
    return layer * case["layers"] + [w]


# ---- inputs --------------------------------------------------------------------------------------------------------------
def _bytes(x, most, dtype):
    """(FP8 bytes, factor): per-tensor scaling, the largest magnitude at the format's largest value."""
    scale = (most / x.abs().amax().float()).reshape(1)
    return (x * scale).clamp(-most, most).to(dtype).view(torch.uint8), scale


def _prepare_adamw(case, gen):
    sizes = _sizes(case)
    padded = [(n + BLOCK - 1) // BLOCK * BLOCK for n in sizes]
    total, count = sum(padded), len(sizes)
    dev = "cuda"

    def flat(dtype, std, of=lambda x: x):
        t = torch.empty(total, dtype=dtype, device=dev)
        for i in range(0, total, 1 << 26):
            t[i:i + (1 << 26)] = of(torch.randn(min(1 << 26, total - i), generator=gen, device=dev).mul_(std))
        # (nothing behind the end of a tensor)
        for piece, n in zip(t.split(padded), sizes):
            piece[n:] = 0
        return t

    def parts(t, unit=1):
        return [x[:-(-n // unit)] for x, n in zip(t.split([p // unit for p in padded]), sizes)]

    s = {"case": case, "p": flat(WIDER[case["param"]], 0.02), "g": flat(WIDER[case["grad"]], 1e-3)}
    m = flat(torch.float32, 3e-4)
    v = flat(torch.float32, 1e-3, lambda x: x.square().add_(1e-7))
    if case["state"] == "fp8":
        for name, x in (("m", m), ("v", v.sqrt_())):
            blocks = x.view(-1, BLOCK)
            scale = 448.0 / blocks.abs().amax(1).clamp(min=1e-20)
            s[name], s[name + "_scale"] = (blocks * scale[:, None]).clamp(-448, 448).to(E4M3).view(-1).view(torch.uint8), scale
        del m, v, x, blocks
    else:
        s["m"], s["v"] = m, v
        del m, v
    s["norm"] = s["g"].float().square().sum(dtype=torch.float64).sqrt().float().reshape(1)
    s["max_norm"] = float(s["norm"]) * (0.3 if case["clips"] else 4.0)
    s["step"] = torch.full((1,), 1000, dtype=torch.int64, device=dev)
    s["lr"] = torch.full((1,), 3e-4, device=dev)
    s["beta1"], s["beta2"], s["eps"] = 0.9, 0.95, 1e-8
    s["seed"] = int(torch.randint(0, 2 ** 62, (1,), generator=gen, device=dev))
    # matrices decay and have copies in FP8; the factor of a copy is from past maxima
    matrix = [n >= case["width"] ** 2 for n in sizes]
    s["weight_decay"] = [0.1 if x else 0.0 for x in matrix]
    if case["copies"]:
        s["q"] = torch.zeros(total, dtype=torch.uint8, device=dev)
        s["q_scale"] = torch.full((count,), 448.0 / 0.125, device=dev)
        s["q_amax"] = torch.zeros(count, device=dev)
        s["qs"] = [x if is_matrix else None for x, is_matrix in zip(parts(s["q"]), matrix)]
    for name in ("p", "g", "m", "v"):
        s[name + "s"] = parts(s[name])
    if case["state"] == "fp8":
        s["m_scales"], s["v_scales"] = parts(s["m_scale"], BLOCK), parts(s["v_scale"], BLOCK)
    # for the plain form: the tensor that a block of BLOCK elements is of, and where that tensor begins
    blocks = torch.tensor([p // BLOCK for p in padded], device=dev)
    s["of"] = torch.repeat_interleave(torch.arange(count, device=dev), blocks)
    s["starts"] = torch.cumsum(blocks, 0) - blocks
    s["decay"], s["is_matrix"] = torch.tensor(s["weight_decay"], device=dev), torch.tensor(matrix, device=dev)
    return s


def _logits(s, dtype):
    x, w = s["A"].view(E4M3).to(dtype), s["B"].view(E4M3).to(dtype)
    return torch.matmul(x, w if s["case"]["weight"] == "in_out" else w.t()) / (s["sA"].to(dtype) * s["sB"].to(dtype))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["kind"] == "adamw":
        return _prepare_adamw(case, gen)
    M, N, K = case["M"], case["N"], case["K"]
    s = {"case": case}
    # logits with a standard deviation of about 2.5
    x = torch.randn((M, K), generator=gen, device="cuda")
    s["A"], s["sA"] = _bytes(x, 448.0, E4M3)
    w = torch.randn((N, K), generator=gen, device="cuda").mul_(2.5 * K ** -0.5)
    s["B"], s["sB"] = _bytes(w, 448.0, E4M3)
    del x, w
    if case["weight"] == "in_out":
        s["B"] = s["B"].t().contiguous()
    # labels over the whole vocabulary, of which a case may hold a piece; some rows (padding, prompts) have none
    labels = torch.randint(0, N if not case["first"] else 8 * N, (M,), generator=gen, device="cuda")
    s["labels"] = torch.where(torch.rand(M, generator=gen, device="cuda") < (0.1 if M > 8 else 0.0), -100, labels)
    if case["kind"] == "loss":
        s["loss"], s["lse"] = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
        # (eight bytes for each row and 32 columns, and for each row)
        s["workspace"] = torch.empty(M * ((N + 31) // 32 + 1) * 8, dtype=torch.uint8, device="cuda")
        return s
    # what the forward pass kept
    s["lse"] = torch.cat([torch.logsumexp(_logits({**s, "A": a}, torch.float32), 1) for a in s["A"].split(max(1, (1 << 28) // N))])
    each = 1.0 / M
    s["dloss"] = torch.rand(M, generator=gen, device="cuda").mul_(each) if case["each_row"] else torch.full((1,), each, device="cuda")
    out = case["out"]
    s["D"] = torch.empty((M, N), dtype=WIDER.get(out, torch.uint8), device="cuda")
    s["sD"] = torch.full((1,), 32768.0 / each, device="cuda") if out == "e5m2" else None
    s["amax"] = torch.zeros(1, device="cuda") if case["amax"] else None
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------
def _result(s):
    case = s["case"]
    if case["kind"] == "loss":
        return {"loss": s["loss"], "lse": s["lse"]}
    if case["kind"] == "loss_grad":
        r = {"out": s["D"].view(E5M2) if case["out"] == "e5m2" else s["D"]}
        return r if s["amax"] is None else {**r, "amax": s["amax"]}
    r = {"p": s["p"]}
    if case["state"] == "fp8":
        r.update(m=s["m"].view(E4M3), v=s["v"].view(E4M3), m_scale=s["m_scale"], v_scale=s["v_scale"])
    else:
        r.update(m=s["m"], v=s["v"])
    if case["copies"]:
        r.update(q=s["q"].view(E4M3), q_amax=s["q_amax"])
    return r


def _run_own(s):
    import paper_2209_05433_amd as fp8
    case = s["case"]
    if case["kind"] == "adamw":
        more = {"m_scale": s["m_scales"], "v_scale": s["v_scales"], "seed": s["seed"]} if case["state"] == "fp8" else {}
        if case["copies"]:
            more.update(q=s["qs"], q_scale=s["q_scale"], q_amax=s["q_amax"])
        fp8.fp8_adamw(s["ps"], s["gs"], s["ms"], s["vs"], s["step"], s["lr"], s["beta1"], s["beta2"], s["eps"], s["weight_decay"],
                      norm=s["norm"], max_norm=s["max_norm"], **more)
        return _result(s)
    out_in = case["weight"] == "out_in"
    if case["kind"] == "loss":
        fp8.fp8_gemm_xent(s["A"], fp8.FP8_E4M3, False, s["B"], fp8.FP8_E4M3, out_in, s["labels"], s["loss"], s["lse"], s["workspace"], s["sA"], s["sB"],
                          first=case["first"], z_weight=case["z_weight"])
        return _result(s)
    out = {"f32": fp8.FP8_OUT_F32, "bf16": fp8.FP8_OUT_BF16, "e5m2": fp8.FP8_OUT_E5M2}[case["out"]]
    fp8.fp8_gemm_xent_grad(s["A"], fp8.FP8_E4M3, False, s["B"], fp8.FP8_E4M3, out_in, s["D"], out, s["sA"], s["sB"], s["labels"], s["lse"], s["dloss"],
                           first=case["first"], z_weight=case["z_weight"], sD=s["sD"], amax_out=s["amax"],
                           flags=fp8.FP8_GEMM_MFMA8 if case["fp8_instructions"] else 0)
    return _result(s)


def _random_bits(s):
    """Philox4x32-10: 32 bits for each element; counter: a tensor's index of four elements (64 bits), the step, the tensor; key: the seed."""
    low = 0xFFFFFFFF
    four = BLOCK // 4
    n = s["of"].numel()
    index = (torch.arange(n, device="cuda") - s["starts"][s["of"]])[:, None] * four + torch.arange(four, device="cuda")
    index = index.view(-1)
    c0, c1, c2, c3 = index & low, index >> 32, (s["step"] & low).expand(index.shape), s["of"].repeat_interleave(four)
    k0, k1 = s["seed"] & low, s["seed"] >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([c0, c1, c2, c3], 1).view(-1)


def _stochastic(x, bits):
    """x rounded to one of its two E4M3 neighbours, away from zero if the part of the gap below it and 16 random bits come to one."""
    y = x.abs().clamp(max=448.0)
    # the gap between its neighbours, 2^(exponent - 3) and 2^-9 at least, from the exponent's bits
    step = ((y.view(torch.int32) >> 23).clamp(min=121) - 3 << 23).view(torch.float32)
    low = torch.floor(y / step) * step
    up = torch.floor((y - low) / step * 65536.0) + bits >= 65536
    return torch.copysign(low + up * step, x)


def _block_factors(x):
    most = x.abs().amax(1, keepdim=True)
    return torch.where((most > 0) & torch.isfinite(448.0 / most), 448.0 / most, torch.ones_like(most))


def _run_adamw_plain(s):
    case = s["case"]
    rows = lambda t: t.view(-1, BLOCK)      # noqa: E731
    states8 = case["state"] == "fp8"
    coefficient = (s["max_norm"] / (s["norm"] + 1e-6)).clamp(max=1.0)
    g = rows(s["g"]).float() * coefficient
    if states8:
        m = rows(s["m"].view(E4M3)).float() * (1.0 / s["m_scale"])[:, None]
        r = rows(s["v"].view(E4M3)).float() * (1.0 / s["v_scale"])[:, None]
        v = r * r
    else:
        m, v = rows(s["m"]), rows(s["v"])
    m = m * s["beta1"] + g * (1 - s["beta1"])
    v = v * s["beta2"] + g * g * (1 - s["beta2"])
    t = s["step"].double()
    c1, c2 = (1 - s["beta1"] ** t).float(), (1 - s["beta2"] ** t).float()
    r = torch.sqrt(v)
    p = rows(s["p"]).float()
    p = p - s["lr"] * (s["decay"][s["of"]][:, None] * p + (m / c1) / (r / torch.sqrt(c2) + s["eps"]))
    if states8:
        bits = rows(_random_bits(s))
        for name, x, b in (("m", m, bits & 0xFFFF), ("v", r, bits >> 16)):
            scale = _block_factors(x)
            code = _stochastic(x * scale, b)
            if name == "v":
                code = torch.where(x > 0, code.clamp(min=2.0 ** -9), code)
            s[name].copy_(code.to(E4M3).view(torch.uint8).view(-1))
            s[name + "_scale"].copy_(scale.view(-1))
    else:
        s["m"].copy_(m.view(-1))
        s["v"].copy_(v.view(-1))
    s["p"].copy_(p.view(-1))
    if case["copies"]:
        # (copies and maxima of the weights as updated, before they are rounded to what they are kept in)
        scaled = (p * s["q_scale"][s["of"]][:, None]).clamp(-448.0, 448.0)
        kept = s["is_matrix"][s["of"]][:, None]
        s["q"].copy_(torch.where(kept, scaled, torch.zeros_like(scaled)).to(E4M3).view(torch.uint8).view(-1))
        s["q_amax"].zero_().scatter_reduce_(0, s["of"], torch.where(kept, p, torch.zeros_like(p)).abs().amax(1), "amax")
    return _result(s)


def _run_plain(s):
    case = s["case"]
    if case["kind"] == "adamw":
        return _run_adamw_plain(s)
    z = _logits(s, torch.float32)
    column = s["labels"] - case["first"]
    here, counts = (column >= 0) & (column < case["N"]) & (s["labels"] >= 0), s["labels"] >= 0
    at = torch.where(here, column, torch.zeros_like(column))[:, None]
    if case["kind"] == "loss":
        top = z.amax(1)
        lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
        loss = lse + case["z_weight"] * lse * lse - torch.where(here, z.gather(1, at)[:, 0], torch.zeros_like(lse))
        s["loss"].copy_(torch.where(counts, loss, torch.zeros_like(loss)))
        s["lse"].copy_(lse)
        return _result(s)
    lse = s["lse"][:, None]
    y = torch.exp(z - lse) * (1 + 2 * case["z_weight"] * lse)
    y.scatter_add_(1, at, -here.float()[:, None])
    y = y * torch.where(counts, s["dloss"], torch.zeros_like(s["dloss"]))[:, None]
    if s["amax"] is not None:
        s["amax"].copy_(y.abs().amax().reshape(1))
    if case["out"] == "e5m2":
        s["D"].copy_((y * s["sD"]).clamp(-57344.0, 57344.0).to(E5M2).view(torch.uint8))
    else:
        s["D"].copy_(y)
    return _result(s)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- in 64 bits -------------------------------------------------------------------------------------------------------------
def _exact_adamw(s):
    case = s["case"]
    lr, t = float(s["lr"]), int(s["step"])
    b1, b2 = s["beta1"], s["beta2"]
    clip = min(1.0, s["max_norm"] / (float(s["norm"]) + 1e-6))
    res = {name: [] for name in ("p", "m", "v", "m_scale", "v_scale", "q")}
    tops = []
    for i in range(len(s["ps"])):
        # (a tensor and the zeros behind it)
        begin = int(s["starts"][i]) * BLOCK
        end = int(s["starts"][i + 1]) * BLOCK if i + 1 < len(s["ps"]) else s["p"].numel()
        g = s["g"][begin:end].double() * clip
        m, v = s["m"][begin:end], s["v"][begin:end]
        if case["state"] == "fp8":
            blocks = slice(begin // BLOCK, end // BLOCK)
            m = (m.view(E4M3).double().view(-1, BLOCK) / s["m_scale"][blocks].double()[:, None]).view(-1)
            v = (v.view(E4M3).double().view(-1, BLOCK) / s["v_scale"][blocks].double()[:, None]).view(-1).square()
        m, v = torch.lerp(g, m.double(), b1), torch.lerp(g.square(), v.double(), b2)
        p = s["p"][begin:end].double()
        p = p * (1 - lr * s["weight_decay"][i]) - lr / (1 - b1 ** t) * m / (v.sqrt() * (1 - b2 ** t) ** -0.5 + s["eps"])
        res["p"].append(p)
        if case["state"] == "fp8":
            for name, x in (("m", m), ("v", v.sqrt())):
                x = x.view(-1, BLOCK)
                scale = 448.0 / torch.linalg.vector_norm(x, math.inf, 1)
                scale[torch.isinf(scale)] = 1.0
                res[name].append((x * scale[:, None]).view(-1))
                res[name + "_scale"].append(scale)
        else:
            res["m"].append(m)
            res["v"].append(v)
        if case["copies"]:
            matrix = s["qs"][i] is not None
            res["q"].append((p * float(s["q_scale"][i])).clamp(-448, 448) if matrix else torch.zeros_like(p))
            tops.append(float(p.abs().max()) if matrix else 0.0)
    res = {name: torch.cat(x) for name, x in res.items() if x}
    if tops:
        res["q_amax"] = torch.tensor(tops, dtype=torch.float64, device="cuda")
    return res


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "adamw":
        return _exact_adamw(s)
    z = _logits(s, torch.float64)
    M, N, w = case["M"], case["N"], case["z_weight"]
    rows = torch.arange(M, device="cuda")
    counts = s["labels"] >= 0
    here = counts & (s["labels"] >= case["first"]) & (s["labels"] < case["first"] + N)
    rows, columns = rows[here], (s["labels"] - case["first"])[here]
    if case["kind"] == "loss":
        lse = torch.logsumexp(z, 1)
        loss = lse + w * lse.square()
        loss[rows] -= z[rows, columns]
        return {"loss": loss.masked_fill(~counts, 0.0), "lse": lse}
    lse = s["lse"].double()[:, None]
    y = z.sub_(lse).exp_().mul_(1 + 2 * w * lse)
    y[rows, columns] -= 1.0
    y *= (s["dloss"].double() * counts)[:, None]
    res = {} if s["amax"] is None else {"amax": y.abs().max().reshape(1)}
    if case["out"] == "e5m2":
        y = (y * float(s["sD"])).clamp(-57344, 57344)
    return {"out": y, **res}


def work(case):
    if case["kind"] == "adamw":
        sizes, width = _sizes(case), {"f32": 4, "bf16": 2}
        n = sum(sizes)
        moved = n * (2 * width[case["param"]] + width[case["grad"]] + (16 if case["state"] == "f32" else 4))
        if case["state"] == "fp8":
            moved += 16 * sum(-(-x // BLOCK) for x in sizes)
        if case["copies"]:
            moved += sum(x for x in sizes if x >= case["width"] ** 2)
        return {"bytes": moved, "flops": 15 * n}
    M, N, K = case["M"], case["N"], case["K"]
    moved = M * K + N * K + 8 * M + 8 * M
    if case["kind"] == "loss_grad":
        moved += M * N * {"f32": 4, "bf16": 2, "e5m2": 1}[case["out"]]
    return {"bytes": moved, "flops": 2 * M * N * K}
