"""Operators around quantised linear layers, as a list of timed cases.

lookup           Y[t] = alpha S[id, c // group] C[code[id, c // d], c % d]: rows of an embedding table kept as packed codes
lookup_gradient  of that: dC (codebook) and dS (group scales, all rows of the table) from dY and the tokens
table            the same of a float32 table, as the quantiser gives it in training: Y[t] = alpha W[id], dW = alpha sum of dY by id
keep             activations kept in 8 bits (a power of two for every 32 of a row) and brought back
kept_gradient    the gradients of a product with a coded layer, its input kept in 8 bits between forward and backward pass
int8             Y = X W^T in 8-bit integers, with a scale for each token and for each of the layer's rows
int8_gradient    dX = dY W through such a layer

Sizes are the package's own layers (512 x 1000 classifier, 3x3 convolutions of 512 channels as matrices, the 4096 x 4096 linear
layer), its bits per weight, and generic token counts and vocabularies.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_context = None


def _lookup(name, n, rows, cols, k, d, group, dtype, kind="lookup"):
    return {"name": name, "kind": kind, "n": n, "rows": rows, "cols": cols, "k": k, "d": d, "group": group, "dtype": dtype}


def _plain(name, kind, n, rows, cols, dtype):
    return {"name": name, "kind": kind, "n": n, "rows": rows, "cols": cols, "dtype": dtype}


def listed():
    return [
        # One decoded token's row of a stored table, 4 bits, scales of groups of 128: latency is all.
        _lookup("lookup_1_k16", 1, 32_000, 4096, 16, 1, 128, "bf16"),
        # A prompt's rows of a table in 8-bit codes of 4-vectors with one scale a row.
        _lookup("lookup_8192_k256d4", 8192, 32_000, 4096, 256, 4, 4096, "f16"),
        # Training the codebook and scales of a stored table on a batch of 8192 tokens, some of them padding.
        _lookup("lookup_gradient_8192_k16", 8192, 32_000, 4096, 16, 1, 128, "bf16", "lookup_gradient"),
        # The same of a small odd table without scales, a codebook that is no power of two, in float32.
        _lookup("lookup_gradient_301_k100d2", 301, 1000, 734, 100, 2, 0, "f32", "lookup_gradient"),
        # A table in training, before it is stored: the forward and backward pass of its lookup beside the quantiser.
        _plain("table_4096_v32000", "table", 4096, 32_000, 1024, "bf16"),
        # A short sequence and a small table, full precision.
        _plain("table_33_v1000", "table", 33, 1000, 512, "f32"),
        # The input of a linear layer kept in 8 bits for a batch of 8192 tokens.
        _plain("keep_8192_4096", "keep", 8192, 0, 4096, "bf16"),
        # Fine-tuning the 4096 x 4096 layer's codebook and scales with inputs kept in 8 bits.
        _lookup("kept_gradient_2048_4096_k16", 2048, 4096, 4096, 16, 1, 128, "bf16", "kept_gradient"),
        # One token through a 4096 x 4096 layer of 8-bit integers: single-token serving, bound by reading the layer.
        _plain("int8_1_4096", "int8", 1, 4096, 4096, "bf16"),
        # Several sequences' tokens through a convolution as a matrix, an odd count.
        _plain("int8_41_conv512", "int8", 41, 512, 4608, "f16"),
        # A prompt of 2048 tokens: bound by the matrix cores.
        _plain("int8_2048_4096", "int8", 2048, 4096, 4096, "bf16"),
        # The gradient of a batch through the 512 x 1000 classifier held in 8-bit integers, on the way to what is trained below it.
        _plain("int8_gradient_1001_fc", "int8_gradient", 1001, 1000, 512, "f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["lookup", "lookup_gradient", "lookup_gradient", "table", "keep", "kept_gradient", "int8", "int8", "int8_gradient"])
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    if kind in ("lookup", "lookup_gradient", "kept_gradient"):
        kept = kind == "kept_gradient"
        d = rng.choice([1, 1, 1, 2, 4, 8])
        k = rng.choice([2, 3, 4, 8, 16, 16, 64] if d == 1 else [4, 16, 100, 256])
        rows, cols = _log(rng, 100, 4096 if kept else 32_000), max(1, _log(rng, 64, 4096) // d) * d
        n = _log(rng, 1, (512 if dtype == "f32" else 2048) if kept else 8192)
        case = _lookup("", n, rows, cols, k, d, rng.choice([0, 32, 64, 128, 128, max(32, cols // 32 * 32)]), dtype, kind)
    elif kind == "table":
        case = _plain("", kind, _log(rng, 1, 4096), _log(rng, 50, 32_000), _log(rng, 16, 1024), dtype)
    elif kind == "keep":
        case = _plain("", kind, _log(rng, 1, 8192 if dtype != "f32" else 4096), 0, _log(rng, 16, 4096), dtype)
    else:
        top = 4096 if kind == "int8" else 2048
        case = _plain("", kind, _log(rng, 1, 2048 if kind == "int8" else 1024), _log(rng, 100, top), _log(rng, 100, top), dtype)
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


def _make_codes(case, g):
    rows, cols, k, d, group = (case[key] for key in ("rows", "cols", "k", "d", "group"))
    m = rows * cols // d
    C = torch.randn(k, d, device="cuda", generator=g)
    if d == 1:  # codes of normal weights: the outer codewords are the rare ones
        C = torch.sort(C, 0).values
        codes = torch.bucketize(torch.randn(m, device="cuda", generator=g), (C[1:, 0] + C[:-1, 0]) / 2)
    else:
        codes = torch.randint(0, k, (m,), device="cuda", generator=g)
    S, std = None, 1.0 / math.sqrt(cols)
    if group:
        S = std * torch.exp(0.25 * torch.randn(rows, _groups(cols, group), device="cuda", generator=g))
    else:
        C = C * std
    codes = codes.to(torch.int32)
    return {"codes": codes, "words": _pack(codes, _bits(k)), "C": C.to(DTYPES[case["dtype"]]), "S": S, "group": group, "rows": rows,
            "cols": cols}


def _make_tokens(n, rows, g):
    """Tokens whose frequency falls with their rank, as a text's do, a fiftieth of them padding."""
    u = torch.rand(n, device="cuda", generator=g, dtype=torch.float64)
    ids = ((u * math.log(rows + 1.0)).exp().long() - 1).clamp(0, rows - 1)
    return torch.where(torch.rand(n, device="cuda", generator=g) < 0.02, torch.full_like(ids, -1), ids)


def _make_activations(n, cols, dtype, g):
    """Columns of different sizes, a few of them much larger than the rest."""
    size = torch.exp(0.5 * torch.randn(cols, device="cuda", generator=g))
    size = torch.where(torch.rand(cols, device="cuda", generator=g) < 0.005, 10.0 * size, size)
    return (torch.randn(n, cols, device="cuda", generator=g) * size).to(dtype)


def _to_int8(x):
    """Rows in 8-bit integers: scale = the row's largest size / 127, to the nearest, ties to even."""
    x = x.float()
    s = (x.abs().amax(1) / 127.0).clamp(min=2.0 ** -126)
    return torch.round(x.double() / s.double()[:, None]).to(torch.int8), s  # a quotient next to a border keeps its side in 64 bits


def _make(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, n, rows, cols, dtype = case["kind"], case["n"], case["rows"], case["cols"], DTYPES[case["dtype"]]
    new = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    state = {"kind": kind, "dtype": dtype}
    if kind in ("lookup", "lookup_gradient", "kept_gradient"):
        state.update(_make_codes(case, g))
    if kind in ("lookup", "lookup_gradient", "table"):
        state["ids"], state["alpha"] = _make_tokens(n, rows, g), math.sqrt(cols)
    if kind == "table":
        state["W"] = new(rows, cols) / math.sqrt(cols)
    if kind in ("lookup_gradient", "table"):
        state["dY"] = (new(n, cols) / math.sqrt(n)).to(dtype)
    if kind in ("keep", "kept_gradient", "int8"):
        state["X"] = _make_activations(n, cols, dtype, g)
    if kind in ("kept_gradient", "int8_gradient"):
        state["dY"] = (new(n, rows) / math.sqrt(n)).to(dtype)
    if kind in ("int8", "int8_gradient"):
        state["W8"], state["scale"] = _to_int8(new(rows, cols) * math.sqrt(2.0 / cols) * torch.exp(0.25 * new(rows, 1)))
    return state


def prepare(case, seed):
    state = _make(case, seed)
    if own:
        from paper_2312_07759_amd import binding
        global _context
        _context = _context or binding.Context(torch.cuda.current_device())
        state["ctx"] = _context
        if "words" in state:  # the layer as a program holds it
            state["layer"] = binding.CodesLayer(state["words"], state["rows"], state["cols"], state["C"], state["S"], state["group"])
        if "W8" in state:
            state["layer"] = binding.Int8Layer(state["W8"], state["scale"], state["dtype"])
    return state


# ------------------------------------------------------------------------------------------------ one pass

def _codes(s, rows):
    """Codes [len(rows), cols / d] of some of the layer's rows, out of the stream."""
    k, d = s["C"].shape
    bits, each = _bits(k), s["cols"] // d
    words = s["words"].long() & 0xFFFFFFFF
    at = (rows[:, None] * each + torch.arange(each, device=words.device)) * bits
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


def _run_lookup(s):
    there, at = s["ids"] >= 0, s["ids"].clamp(min=0)
    Y = s["C"].float()[_codes(s, at)].view(len(at), -1)
    if s["S"] is not None:
        Y = Y * _spread(s["S"][at], s["cols"], s["group"])
    return (Y * (s["alpha"] * there)[:, None]).to(s["dtype"])


def _run_lookup_gradient(s):
    there, at, (k, d) = s["ids"] >= 0, s["ids"].clamp(min=0), s["C"].shape
    codes = _codes(s, at)
    G = s["dY"].float() * (s["alpha"] * there)[:, None]
    out, SG = {}, G
    if s["S"] is not None:
        w = s["C"].float()[codes].view_as(G)
        out["dS"] = torch.zeros_like(s["S"]).index_add_(0, at, _per_group(G * w, s["group"]))
        SG = G * _spread(s["S"][at], s["cols"], s["group"])
    place = (torch.arange(len(at), device=at.device)[:, None] * k + codes).view(-1)
    bins = torch.zeros(len(at) * k, d, device=at.device).index_add_(0, place, SG.view(-1, d))  # token by token, then over the tokens
    out["dC"] = bins.view(-1, k, d).double().sum(0).float()
    return out


def _run_table(s):
    there, at = s["ids"] >= 0, s["ids"].clamp(min=0)
    by = (s["alpha"] * there)[:, None].float()
    return {"Y": (s["W"][at] * by).to(s["dtype"]), "dW": torch.zeros_like(s["W"]).index_add_(0, at, s["dY"].float() * by)}


def _kept(X):
    """X as 8 bits hold it: integers of up to 127 times a power of two, one for every 32 elements of a row."""
    n, cols = X.shape
    top = math.frexp(torch.finfo(X.dtype).max)[1]
    x = torch.nn.functional.pad(X, (0, -cols % 32)).double().view(n, -1, 32)
    size = x.abs().amax(2, keepdim=True)
    exponent = torch.frexp(size)[1].clamp(min=-125)  # size < 2^exponent
    step = (exponent.long() - 7 + 1023 << 52).view(torch.float64)  # 2^(exponent - 7), which half the quotients' ties depend on
    step = torch.where((size >= 127.5 * step) & (exponent < top), 2 * step, step)
    return (torch.round(x / step).clamp(-127, 127) * step).view(n, -1)[:, :cols].to(X.dtype)


def _run_kept_gradient(s):
    (k, d), rows, cols = s["C"].shape, s["rows"], s["cols"]
    codes = _codes(s, torch.arange(rows, device=s["dY"].device))
    unscaled = s["C"].float()[codes].view(rows, cols)
    X, dY = _kept(s["X"]).float(), s["dY"].float()
    out = {}
    P = dY.t() @ X
    SP, W = P, unscaled
    if s["S"] is not None:
        scales = _spread(s["S"], cols, s["group"])
        out["dS"] = _per_group(P * unscaled, s["group"])
        SP, W = P * scales, unscaled * scales
    out["dX"] = (dY @ W).to(s["dtype"])
    place = (torch.arange(rows, device=codes.device)[:, None] * k + codes).view(-1)
    bins = torch.zeros(rows * k, d, device=codes.device).index_add_(0, place, SP.view(-1, d))  # row by row, then over the rows
    out["dC"] = bins.view(rows, k, d).double().sum(0).float()
    return out


def _run_int8(s):
    q, scale = _to_int8(s["X"])
    return (q.float() @ s["W8"].float().t() * scale[:, None] * s["scale"]).to(s["dtype"])


def _run_int8_gradient(s):
    return (s["dY"].float() @ (s["W8"].float() * s["scale"][:, None])).to(s["dtype"])


def run(state):
    s = state
    if not own:
        return {"lookup": _run_lookup, "lookup_gradient": _run_lookup_gradient, "table": _run_table, "keep": lambda s: _kept(s["X"]),
                "kept_gradient": _run_kept_gradient, "int8": _run_int8, "int8_gradient": _run_int8_gradient}[s["kind"]](s)
    ctx = s["ctx"]
    if s["kind"] == "lookup":
        return ctx.codes_embedding(s["layer"], s["ids"], s["alpha"])
    if s["kind"] == "lookup_gradient":
        return ctx.codes_embedding_backward(s["layer"], s["ids"], s["dY"], s["alpha"])
    if s["kind"] == "table":
        return {"Y": ctx.embedding(s["W"], s["ids"], s["alpha"], s["dtype"]),
                "dW": ctx.embedding_backward(s["dY"], s["ids"], s["W"].shape[0], s["alpha"])}
    if s["kind"] == "keep":
        return ctx.restore8(ctx.keep8(s["X"]))
    if s["kind"] == "kept_gradient":
        return ctx.codes_linear_backward(s["layer"], ctx.keep8(s["X"]), s["dY"])
    if s["kind"] == "int8":
        return ctx.int8_linear(s["layer"], s["X"])
    return ctx.int8_linear_backward(s["layer"], s["dY"])


# ------------------------------------------------------------------------------------------------ work and values

def _distinct(n, rows):
    """Different tokens that n of _make_tokens are expected to hold."""
    p = torch.log1p(1.0 / torch.arange(1, rows + 1, dtype=torch.float64)) / math.log(rows + 1.0)
    return float((-torch.expm1(n * torch.log1p(-p))).sum())


def work(case):
    kind, n, rows, cols = (case[key] for key in ("kind", "n", "rows", "cols"))
    width = 4 if case["dtype"] == "f32" else 2
    if kind == "keep":  # the activations, their 8 bits and exponents written and read, the activations brought back
        return {"bytes": n * cols * (2 * width + 2 + 2 / 32), "flops": 4 * n * cols}
    if kind == "table":
        return {"bytes": 4 * cols * (_distinct(n, rows) + rows) + 2 * n * cols * width + 16 * n, "flops": 2 * n * cols}
    if kind == "int8":
        return {"bytes": rows * cols + 4 * rows + n * width * (rows + cols), "flops": 2 * n * rows * cols}
    if kind == "int8_gradient":
        return {"bytes": rows * cols + 4 * rows + n * width * (rows + cols), "flops": 2 * n * rows * cols}
    k, d, groups = case["k"], case["d"], _groups(cols, case["group"])
    row = cols // d * _bits(k) / 8 + 4 * groups
    if kind == "kept_gradient":  # .. and the input read, its 8 bits written and read
        layer = rows * row + width * k * d
        return {"bytes": layer + n * (width * (rows + 2 * cols) + 2 * cols) + 4 * k * d + 4 * rows * groups, "flops": 4 * n * rows * cols}
    read = _distinct(n, rows) * row + width * k * d + 8 * n + n * width * cols
    if kind == "lookup":
        return {"bytes": read, "flops": 2 * n * cols}
    return {"bytes": read + 4 * k * d + 4 * rows * groups, "flops": 4 * n * cols}


def _wide_layer(s):
    """Codes [rows, cols / d], and in 64 bits the codewords and the scales in the places of the weights (scales None: none)."""
    rows, cols = s["rows"], s["cols"]
    codes = s["codes"].long().reshape(rows, -1)
    unscaled = s["C"].double()[codes].reshape(rows, cols)
    wide = None
    if s["S"] is not None:
        wide = s["S"].double()[:, torch.arange(cols, device=codes.device) // s["group"]]
    return codes, unscaled, wide


def _layer_gradients(s, P):
    """dC and dS from P = the gradient in the scaled weights, in 64 bits."""
    codes, unscaled, wide = _wide_layer(s)
    cols, (k, d) = s["cols"], s["C"].shape
    out = {}
    if wide is not None:
        out["dS"] = torch.stack([(P[:, c:c + s["group"]] * unscaled[:, c:c + s["group"]]).sum(1) for c in range(0, cols, s["group"])], 1)
        P = P * wide
    P, codes = P.reshape(-1, d), codes.reshape(-1)
    out["dC"] = torch.stack([(P * (codes == j).double()[:, None]).sum(0) for j in range(k)])
    return out


def _by_token(s, rows):
    """Sums of dY by token, in 64 bits: [rows, cols]."""
    ids, held = s["ids"], s["ids"] >= 0
    sums = torch.zeros(rows, s["dY"].shape[1], dtype=torch.float64, device=ids.device)
    return sums.index_put_((ids[held],), s["dY"][held].double() * s["alpha"], accumulate=True)


def _exact_kept(X):
    """What 8 bits keep of X, in 64 bits."""
    X, limit = X.double(), torch.finfo(X.dtype).max
    out = torch.zeros_like(X)
    power = torch.tensor([2.0 ** i for i in range(-126, 129)], dtype=torch.float64, device=X.device)
    for c in range(0, X.shape[1], 32):
        block = X[:, c:c + 32]
        size = block.abs().max(1, keepdim=True).values
        low = (torch.bucketize(size, power, right=True) - 1).clamp(min=0)  # power[low] <= size < power[low + 1]
        step = power[low] / 64
        step = torch.where((torch.round(size / step) <= 127) | (power[low + 1] > limit), step, 2 * step)
        out[:, c:c + 32] = torch.round(block / step).clamp(-127, 127) * step
    return out


def exact(case, seed):
    s, kind = _make(case, seed), case["kind"]
    rows, cols = case["rows"], case["cols"]
    if kind == "keep":
        return _exact_kept(s["X"])
    if kind == "table":
        padded = torch.cat([s["W"].double() * s["alpha"], torch.zeros(1, cols, dtype=torch.float64, device=s["W"].device)])
        return {"Y": padded[s["ids"]], "dW": _by_token(s, rows)}  # token -1 is the row of zeros behind the last
    if kind == "lookup":
        codes, unscaled, wide = _wide_layer(s)
        Y = s["alpha"] * (unscaled if wide is None else unscaled * wide)[s["ids"]]
        Y[s["ids"] < 0] = 0
        return Y
    if kind == "lookup_gradient":
        return _layer_gradients(s, _by_token(s, rows))
    if kind == "int8_gradient":
        return s["dY"].double() @ (s["W8"].double() * s["scale"].double()[:, None])
    if kind == "int8":
        X = s["X"].double()
        step = (s["X"].float().abs().max(1).values / 127).double()[:, None]  # the scale is a float32 number
        below = torch.floor(X / step)
        over = X - below * step - step / 2  # which of the two integers around it is nearer; the even one of a tie
        up = (over > 0) | ((over == 0) & (below % 2 != 0))
        return (below + up) * step @ (s["W8"].double() * s["scale"].double()[:, None]).t()
    codes, unscaled, wide = _wide_layer(s)
    dY = s["dY"].double()
    out = _layer_gradients(s, dY.t() @ _exact_kept(s["X"]))
    out["dX"] = dY @ (unscaled if wide is None else unscaled * wide)
    return out
