"""Operators on quantised linear layers and their training, as a list of timed cases.

product   Y = X W^T of a layer kept as packed codes: w[n, c] = S[n, c // group] C[code[n, c // d], c % d]
gradient  of that product: dX, dC (codebook) and dS (group scales)
scale     a layer divided by its groups' root mean squares before clustering, multiplied by them after it, and the gradients
distill   Kullback-Leibler loss against a teacher's top logits, and its gradient

Sizes are the package's own layers (512 x 1000 classifier, 3x3 convolutions of 256 and 512 channels as matrices, the 4096 x
4096 linear layer), its bits per weight, and generic token counts and vocabularies.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_context = None


def _product(name, n, rows, cols, k, d, group, dtype, kind="product"):
    return {"name": name, "kind": kind, "n": n, "rows": rows, "cols": cols, "k": k, "d": d, "group": group, "dtype": dtype}


def _distill(name, n, vocab, top, tau, dtype):
    return {"name": name, "kind": "distill", "n": n, "vocab": vocab, "top": top, "tau": tau, "dtype": dtype}


def listed():
    return [
        # The quantised classifier on one input, codes of 2 bits, no scales: latency is all.
        _product("product_1_fc_k4", 1, 1000, 512, 4, 1, 0, "f32"),
        # One token through a 4096 x 4096 layer at 4 bits with a scale for every 128 weights: single-token serving.
        _product("product_1_4096_k16", 1, 4096, 4096, 16, 1, 128, "bf16"),
        # A small odd batch of decoding tokens, 8-bit codes of 4-vectors, one scale a row (a convolution as a matrix).
        _product("product_7_conv512_k256d4", 7, 512, 4608, 256, 4, 4608, "f16"),
        # Several sequences' tokens at once, 3 bits, short groups: between the matrix-vector and the matrix product.
        _product("product_61_4096_k8", 61, 4096, 4096, 8, 1, 64, "bf16"),
        # A prompt of 2048 tokens through the same layer: bound by the matrix cores.
        _product("product_2048_4096_k16", 2048, 4096, 4096, 16, 1, 128, "bf16"),
        # Fine-tuning the codebook and scales of that layer on a batch of 2048 tokens.
        _product("gradient_2048_4096_k16", 2048, 4096, 4096, 16, 1, 128, "bf16", "gradient"),
        # The same for a convolution as a matrix, vector codes, no scales, an odd number of rows of a batch, in float32.
        _product("gradient_1001_conv512_k256d4", 1001, 512, 4608, 256, 4, 0, "f32", "gradient"),
        # Scales of the 4096 x 4096 layer, 128 weights a group, one training step's way there and back.
        {"name": "scale_4096_g128", "kind": "scale", "rows": 4096, "cols": 4096, "group": 128},
        # The classifier's with a group that does not divide its rows.
        {"name": "scale_fc_g96", "kind": "scale", "rows": 1000, "cols": 512, "group": 96},
        # A batch of 2048 tokens against a teacher's 64 largest of 128000 logits.
        _distill("distill_2048_v128000", 2048, 128_000, 64, 2.0, "bf16"),
        # A short sequence, an odd vocabulary, full precision: few rows, so each has to be spread over the device.
        _distill("distill_5_v50001", 5, 50_001, 20, 1.0, "f32"),
        # A classifier's 1000 classes and the teacher's five best.
        _distill("distill_256_v1000", 256, 1_000, 5, 4.0, "f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["product", "product", "product", "gradient", "gradient", "scale", "distill", "distill"])
    if kind == "scale":
        rows, cols = _log(rng, 16, 4096), _log(rng, 64, 4608)
        return {"kind": "scale", "rows": rows, "cols": min(cols, 16_777_216 // rows), "group": rng.choice([32, 64, 96, 128, cols])}
    if kind == "distill":
        vocab = _log(rng, 1_000, 128_000)
        case = _distill("", min(_log(rng, 1, 2048), 200_000_000 // vocab), vocab, rng.choice([1, 5, 20, 64, 100]),
                        rng.choice([1.0, 2.0, 4.0]), rng.choice(["f32", "f16", "bf16"]))
    else:
        d = rng.choice([1, 1, 1, 2, 4, 8])
        k = rng.choice([2, 3, 4, 8, 16, 16, 64] if d == 1 else [4, 16, 100, 256])
        rows, cols = _log(rng, 100, 4096), max(1, _log(rng, 200, 4608) // d) * d
        dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
        n = _log(rng, 1, 512 if dtype == "f32" else 2048)
        case = _product("", n, rows, min(cols, 4096 * 4096 // rows // d * d), k, d, rng.choice([0, 32, 64, 128, 128, cols // 32 * 32]),
                        dtype, kind)
    case.pop("name")
    return case


# ------------------------------------------------------------------------------------------------ inputs

def _bits(k):
    return max(1, (k - 1).bit_length())


def _groups(cols, group):
    return -(-cols // group) if group else 0


def _pack(codes, bits):
    """Codes as one little-endian stream of `bits` bits each, in 32-bit words."""
    words = torch.zeros(-(-codes.numel() * bits // 32) * 32, dtype=torch.uint8, device=codes.device)
    stream = words[: codes.numel() * bits].view(-1, bits)
    for t in range(bits):
        stream[:, t] = (codes >> t) & 1
    weight = 1 << torch.arange(8, device=codes.device, dtype=torch.int32)
    return (words.view(-1, 8) * weight).sum(1).to(torch.uint8).view(torch.int32)


def _make_product(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, rows, cols, k, d, group = (case[key] for key in ("n", "rows", "cols", "k", "d", "group"))
    dtype = DTYPES[case["dtype"]]
    m = rows * cols // d
    C = torch.randn(k, d, device="cuda", generator=g)
    if d == 1:  # codes of normal weights: the outer codewords are the rare ones
        C = torch.sort(C, 0).values
        codes = torch.bucketize(torch.randn(m, device="cuda", generator=g), (C[1:, 0] + C[:-1, 0]) / 2)
    else:
        codes = torch.randint(0, k, (m,), device="cuda", generator=g)
    std = math.sqrt(2.0 / cols)
    S = None
    if group:
        S = std * torch.exp(0.25 * torch.randn(rows, _groups(cols, group), device="cuda", generator=g))
    else:
        C = C * std
    state = {"kind": case["kind"], "codes": codes.to(torch.int32), "words": _pack(codes, _bits(k)), "C": C.to(dtype), "S": S,
             "group": group, "rows": rows, "cols": cols, "X": torch.randn(n, cols, device="cuda", generator=g).to(dtype)}
    if case["kind"] == "gradient":
        state["dY"] = (torch.randn(n, rows, device="cuda", generator=g) / math.sqrt(n)).to(dtype)
    return state


def _make_scale(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols, group = case["rows"], case["cols"], case["group"]
    new = lambda std: std * torch.randn(rows, cols, device="cuda", generator=g)  # noqa: E731
    W = new(math.sqrt(2.0 / cols))
    return {"kind": "scale", "W": W, "Zq": new(1.0), "dWq": new(1e-2), "dZ": new(1e-4), "group": group}


def _make_distill(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, vocab, top = case["n"], case["vocab"], min(case["top"], case["vocab"])
    gaps = torch.randint(1, max(2, vocab // top), (n, top), device="cuda", generator=g)
    index = (torch.cumsum(gaps, 1) - 1).to(torch.int32)  # distinct
    teacher = 10.0 - 1.5 * torch.rand(n, top, device="cuda", generator=g).cumsum(1)
    logits = 2.5 * torch.randn(n, vocab, device="cuda", generator=g)
    logits.scatter_(1, index.long(), teacher + torch.randn(n, top, device="cuda", generator=g))
    # lists that end early, and positions that do not count (padding, prompts): nothing of the list is valid
    length = torch.randint(0, top + 1, (n, 1), device="cuda", generator=g)
    length = torch.where(torch.rand(n, 1, device="cuda", generator=g) < 0.8, torch.full_like(length, top), length)
    index = torch.where(torch.arange(top, device="cuda") < length, index, torch.full_like(index, -1))
    dloss = torch.rand(n, device="cuda", generator=g) / n
    return {"kind": "distill", "logits": logits.to(DTYPES[case["dtype"]]), "index": index, "teacher": teacher, "tau": case["tau"],
            "dloss": dloss}


def prepare(case, seed):
    if case["kind"] == "scale":
        state = _make_scale(case, seed)
    elif case["kind"] == "distill":
        state = _make_distill(case, seed)
    else:
        state = _make_product(case, seed)
    if own:
        from paper_2312_07759_amd import binding
        global _context
        _context = _context or binding.Context(torch.cuda.current_device())
        state["ctx"] = _context
        if "words" in state:  # the layer as a program holds it
            state["layer"] = binding.CodesLayer(state["words"], state["rows"], state["cols"], state["C"], state["S"], state["group"])
    return state


# ------------------------------------------------------------------------------------------------ one pass

def _codes(s):
    """The layer's codes, out of the stream."""
    k, d = s["C"].shape
    bits = _bits(k)
    words = s["words"].long() & 0xFFFFFFFF
    at = torch.arange(s["rows"] * s["cols"] // d, device=words.device) * bits
    low = at >> 5
    pair = words[low] | (words[(low + 1).clamp(max=words.numel() - 1)] << 32)
    return (pair >> (at & 31)) & ((1 << bits) - 1)


def _spread(S, cols, group):
    return S.repeat_interleave(group, 1)[:, :cols]


def _per_group(v, group):
    """Sums over the groups of each row, the last one shorter."""
    rows, cols = v.shape
    whole = cols // group * group
    sums = v[:, :whole].view(rows, -1, group).sum(2)
    return sums if whole == cols else torch.cat([sums, v[:, whole:].sum(1, keepdim=True)], 1)


def _run_product(s):
    unscaled = s["C"].float()[_codes(s)].view(s["rows"], s["cols"])
    W = unscaled if s["S"] is None else unscaled * _spread(s["S"], s["cols"], s["group"])
    return (s["X"].float() @ W.t()).to(s["X"].dtype)


def _run_gradient(s):
    codes, (k, d), rows, cols = _codes(s), s["C"].shape, s["rows"], s["cols"]
    unscaled = s["C"].float()[codes].view(rows, cols)
    X, dY = s["X"].float(), s["dY"].float()
    out = {}
    P = dY.t() @ X
    SP, W = P, unscaled
    if s["S"] is not None:
        scales = _spread(s["S"], cols, s["group"])
        out["dS"] = _per_group(P * unscaled, s["group"])
        SP, W = P * scales, unscaled * scales
    out["dX"] = (dY @ W).to(s["X"].dtype)
    place = torch.arange(rows, device=codes.device).repeat_interleave(cols // d) * k + codes
    bins = torch.zeros(rows * k, d, device=codes.device).index_add_(0, place, SP.view(-1, d))  # row by row, then over the rows
    out["dC"] = bins.view(rows, k, d).double().sum(0).float()
    return out


def _run_scale(s):
    W, group = s["W"], s["group"]
    rows, cols = W.shape
    count = _per_group(torch.ones_like(W), group)
    S = (_per_group(W * W, group) / count).sqrt()
    wide = _spread(S, cols, group)
    Z = torch.where(wide > 0, W / wide, torch.zeros_like(W))
    Wq = s["Zq"] * wide
    dZq = s["dWq"] * wide
    dS = _per_group(s["dWq"] * s["Zq"], group)
    inner = (dS - _per_group(s["dZ"] * Z, group) / S) / count
    dW = torch.where(wide > 0, s["dZ"] / wide + Z * _spread(inner, cols, group), torch.zeros_like(W))
    return {"S": S, "Z": Z, "Wq": Wq, "dZq": dZq, "dS": dS, "dW": dW}


def _run_distill(s):
    index, tau = s["index"], s["tau"]
    valid = index >= 0
    some = valid.any(1, keepdim=True)
    t = torch.where(valid, s["teacher"] / tau, torch.full_like(s["teacher"], -math.inf))
    t = t - torch.where(some, t.amax(1, keepdim=True), torch.zeros_like(t[:, :1]))
    total = t.exp().sum(1, keepdim=True)
    p = t.exp() / torch.where(some, total, torch.ones_like(total))
    z = s["logits"].float() / tau
    top = z.amax(1, keepdim=True)
    lse = top + (z - top).exp().sum(1, keepdim=True).log()
    at = index.clamp(min=0).long()
    logp = torch.where(valid, t - total.log(), torch.zeros_like(t))
    loss = (p * (logp - (z.gather(1, at) - lse))).sum(1)
    scale = s["dloss"][:, None] / tau
    dz = (z - lse).exp() * (scale * some)
    dz.scatter_add_(1, at, -p * scale)
    return {"loss": loss, "lse": lse[:, 0], "dlogits": dz.to(s["logits"].dtype)}


def run(state):
    s = state
    if not own:
        return {"product": _run_product, "gradient": _run_gradient, "scale": _run_scale, "distill": _run_distill}[s["kind"]](s)
    ctx = s["ctx"]
    if s["kind"] == "product":
        return ctx.codes_linear(s["layer"], s["X"])
    if s["kind"] == "gradient":
        return ctx.codes_linear_backward(s["layer"], s["X"], s["dY"])
    if s["kind"] == "scale":
        S, Z = ctx.group_scale(s["W"], s["group"])
        Wq = ctx.group_unscale(s["Zq"], S, s["group"])
        dZq, dS = ctx.group_unscale_backward(s["dWq"], s["Zq"], S, s["group"])
        return {"S": S, "Z": Z, "Wq": Wq, "dZq": dZq, "dS": dS, "dW": ctx.group_scale_backward(Z, S, s["group"], s["dZ"], dS)}
    loss, lse, dlogits = ctx.distill(s["logits"], s["index"], s["teacher"], s["tau"], s["dloss"])
    return {"loss": loss, "lse": lse, "dlogits": dlogits}


# ------------------------------------------------------------------------------------------------ work and values

def work(case):
    if case["kind"] == "scale":
        size, scales = case["rows"] * case["cols"], case["rows"] * _groups(case["cols"], case["group"])
        return {"bytes": 4 * (8 * size + 2 * scales), "flops": 14 * size}  # W, Zq, dWq, dZ in; Z, Wq, dZq, dW, S, dS out
    if case["kind"] == "distill":
        size = case["n"] * case["vocab"]
        width = 4 if case["dtype"] == "f32" else 2
        return {"bytes": 2 * width * size + case["n"] * (8 * case["top"] + 12), "flops": 8 * size}
    n, rows, cols, k, d = (case[key] for key in ("n", "rows", "cols", "k", "d"))
    width = 4 if case["dtype"] == "f32" else 2
    layer = rows * cols // d * _bits(k) / 8 + width * k * d + 4 * rows * _groups(cols, case["group"])
    if case["kind"] == "product":
        return {"bytes": layer + width * n * (rows + cols), "flops": 2 * n * rows * cols}
    out = width * n * cols + 4 * k * d + 4 * rows * _groups(cols, case["group"])
    return {"bytes": layer + width * n * (rows + cols) + out, "flops": 4 * n * rows * cols}


def exact(case, seed):
    kind = case["kind"]
    if kind == "scale":
        s = _make_scale(case, seed)
        W, Zq, dWq, dZ = (s[key].double() for key in ("W", "Zq", "dWq", "dZ"))
        rows, cols = W.shape
        group, groups = case["group"], _groups(cols, case["group"])
        member = torch.zeros(groups, cols, dtype=torch.float64, device=W.device)  # which column belongs to which group
        member[torch.arange(cols, device=W.device) // group, torch.arange(cols, device=W.device)] = 1
        count = member.sum(1)
        S = torch.sqrt(W.square() @ member.t() / count)
        Z = W / (S @ member)
        dS = (dWq * Zq) @ member.t()
        dW = dZ / (S @ member) + Z * (((dS - (dZ * Z) @ member.t() / S) / count) @ member)
        return {"S": S, "Z": Z, "Wq": Zq * (S @ member), "dZq": dWq * (S @ member), "dS": dS, "dW": dW}
    if kind == "distill":
        s = _make_distill(case, seed)
        z, tau = s["logits"].double() / case["tau"], case["tau"]
        logq = torch.log_softmax(z, 1)
        p = torch.zeros_like(z)
        entropy = torch.zeros(z.shape[0], dtype=torch.float64, device=z.device)
        for i in range(z.shape[0]):
            held = s["index"][i] >= 0
            if bool(held.any()):
                logp = torch.log_softmax(s["teacher"][i][held].double() / tau, 0)
                p[i, s["index"][i][held].long()] = logp.exp()
                entropy[i] = (logp.exp() * logp).sum()
        q = logq.exp() * (p.sum(1, keepdim=True) > 0)
        return {"loss": entropy - (p * logq).sum(1), "lse": torch.logsumexp(z, 1),
                "dlogits": (q - p) * s["dloss"].double()[:, None] / tau}
    s = _make_product(case, seed)
    rows, cols = case["rows"], case["cols"]
    unscaled = s["C"].double()[s["codes"].long()].reshape(rows, cols)
    wide = 1.0
    if s["S"] is not None:
        wide = s["S"].double()[:, torch.arange(cols, device=unscaled.device) // case["group"]]
    X = s["X"].double()
    if kind == "product":
        return X @ (unscaled * wide).t()
    dY = s["dY"].double()
    P = dY.t() @ X
    out = {"dX": dY @ (unscaled * wide)}
    if s["S"] is not None:
        out["dS"] = torch.stack([(P * unscaled)[:, c:c + case["group"]].sum(1) for c in range(0, cols, case["group"])], 1)
    SP, codes = (P * wide).reshape(-1, case["d"]), s["codes"].long()
    out["dC"] = torch.stack([(SP * (codes == j).double()[:, None]).sum(0) for j in range(case["k"])])
    return out
