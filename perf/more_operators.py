"""A product in 8-bit integers and a gated linear layer, as they are timed.

A Conformer's convolution module begins with a gated linear unit, and gated feed-forward modules take the place of plain ones: two projections
of the same frames, g = x Wg^T + bg and u = x Wu^T + bu, and h = act(g) u.  It is trained with operands in bf16 and sums in 32 bits, and it and the layers
beside it are served in 8-bit integers, with a scale for every frame and every channel.  The cases are single uses of these: one frame of a stream, some
streams together, an ordinary batch of frames (8192 of them, layers of 1024 <-> 4096 as in the repository's benchmark), large and ragged ones.

8 bits: a row's scale is its largest magnitude over 127, in 32 bits, and its codes are the whole numbers nearest to x / scale, ties to even.

The forward pass of a training step keeps the slopes of h, dh/du = act(g) and dh/dg = u act'(g), in bf16; on the way back dg = dh (dh/dg) and
du = dh (dh/du) are rounded to bf16, as operands of the products are.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
WIDTH = {"f32": 4, "bf16": 2}
GATES = ("sigmoid", "swish", "gelu")
MOST_ROUND = 16384 * 8192
MOST_LINEAR = 16384 * 8192 * 8192
MOST_GATED = 8192 * 4096 * 2048


def listed():
    return [
        # a layer's weights on their way into 8 bits, a scale for every column: a matrix of odd sizes
        {"name": "round_channels_ragged", "what": "round", "rows": 971, "cols": 243, "pad": 0, "type": "f32", "columns": True},
        # all of a large batch's activations, a scale for every frame
        {"name": "round_frames_large", "what": "round", "rows": 16384, "cols": 8192, "pad": 0, "type": "bf16", "columns": False},
        # one frame of a streaming encoder through a feed-forward layer's 8-bit weights: latency
        {"name": "linear_frame", "what": "linear", "M": 1, "N": 4096, "K": 1024, "pad": 0, "type": "bf16", "out": "bf16", "bias": True},
        # some streams served together, sizes off the tiles, input a slice of a wider buffer
        {"name": "linear_streams_ragged", "what": "linear", "M": 29, "N": 8200, "K": 971, "pad": 3, "type": "f32", "out": "f32", "bias": False},
        # the largest product
        {"name": "linear_large", "what": "linear", "M": 16384, "N": 8192, "K": 8192, "pad": 0, "type": "bf16", "out": "bf16", "bias": False},
        # one frame through a gated layer as it is trained
        {"name": "gated_frame", "what": "gated", "M": 1, "N": 2048, "K": 512, "pad": 0, "type": "bf16", "weights": "bf16", "out": "bf16", "bias": True, "gate": "sigmoid", "keep": False},
        # a short batch through a gated layer of odd sizes, in fp32 on both sides
        {"name": "gated_ragged", "what": "gated", "M": 1003, "N": 971, "K": 243, "pad": 1, "type": "f32", "weights": "f32", "out": "f32", "bias": True, "gate": "gelu", "keep": True},
        # forward pass of a training step, ordinary batch
        {"name": "gated_batch", "what": "gated", "M": 8192, "N": 4096, "K": 1024, "pad": 0, "type": "bf16", "weights": "bf16", "out": "bf16", "bias": True, "gate": "swish", "keep": True},
        # backward through the small layer of odd sizes
        {"name": "gated_grad_ragged", "what": "gated_backward", "M": 1003, "N": 971, "K": 243, "pad": 1, "type": "f32", "weights": "f32", "out": "f32", "bias": True, "gate": "gelu"},
        # backward pass of a training step, ordinary batch
        {"name": "gated_grad_batch", "what": "gated_backward", "M": 8192, "N": 4096, "K": 1024, "pad": 0, "type": "bf16", "weights": "bf16", "out": "bf16", "bias": True, "gate": "swish"},
        # some streams through a gated layer's 8-bit weights
        {"name": "gated_i8_streams", "what": "gated_i8", "M": 16, "N": 4096, "K": 1024, "pad": 0, "type": "bf16", "out": "bf16", "bias": True, "gate": "swish"},
        # a batch of recorded speech through the same
        {"name": "gated_i8_batch", "what": "gated_i8", "M": 8192, "N": 4096, "K": 1024, "pad": 0, "type": "bf16", "out": "bf16", "bias": True, "gate": "swish"},
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Any size between the listed ones' least and most; half of the widths are whole blocks of 32, a quarter of the inputs slices."""
    what = rng.choice(("round", "linear", "linear", "gated", "gated", "gated_backward", "gated_backward", "gated_i8"))
    while True:
        def wide(lo, hi):
            n = _between(rng, lo, hi)
            return max(32, n // 32 * 32) if rng.random() < 0.5 else n
        case = {"what": what, "pad": rng.randint(1, 64) if rng.random() < 0.25 else 0, "type": rng.choice(("bf16", "bf16", "f32"))}
        if what == "round":
            case |= {"rows": _between(rng, 1, 16384), "cols": wide(32, 8192), "columns": rng.random() < 0.5}
            size, most = case["rows"] * case["cols"] * WIDTH[case["type"]], MOST_ROUND * 2
        else:
            case |= {"M": _between(rng, 1, 16384 if what == "linear" else 8192), "N": wide(64, 8192), "K": wide(64, 8192), "out": rng.choice(("bf16", "f32")), "bias": rng.random() < 0.5}
            if what != "linear":
                case |= {"gate": rng.choice(GATES)}
            if what in ("gated", "gated_backward"):
                case |= {"weights": rng.choice(("bf16", "bf16", "f32"))}
            if what == "gated":
                case |= {"keep": rng.random() < 0.5}
            size, most = case["M"] * case["N"] * case["K"], MOST_LINEAR if what == "linear" else MOST_GATED
        if size <= most:
            return case


# ---- inputs --------------------------------------------------------------------------------------------------------

def _frames(g, rows, cols, pad, kind, spread):
    """Activations: channels of different sizes and offsets; of a batch, the last frames of some utterances are padding (zeros)."""
    size = torch.exp(0.5 * torch.randn(cols, device="cuda", generator=g))
    x = torch.randn(rows, cols + pad, device="cuda", generator=g)
    x[:, :cols] *= size * spread
    x[:, :cols] += torch.randn(cols, device="cuda", generator=g) * (0.3 * spread)
    if rows >= 64:
        x[torch.rand(rows, device="cuda", generator=g) < 0.02] = 0.0
    return x.to(TYPES[kind])[:, :cols]


def _weights(g, rows, cols, kind):
    return (torch.randn(rows, cols, device="cuda", generator=g) * (0.7 / math.sqrt(cols))).to(TYPES[kind])


def _weights_i8(g, rows, cols):
    """A weight matrix's codes (rows padded with zeros to whole 128s) and its channels' scales, in the layout that the products take."""
    w = _weights(g, rows, cols, "f32")
    scales = w.abs().amax(1) / 127.0
    codes = torch.zeros(rows, -(-cols // 128) * 128, device="cuda", dtype=torch.int8)
    codes[:, :cols] = torch.round(w.double() / scales.double()[:, None]).to(torch.int8)
    return codes.view(torch.uint8), scales


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    what, kind = case["what"], case["type"]
    s = {"case": case, "what": what}

    def empty(rows, cols, t):
        return torch.empty(rows, cols, device="cuda", dtype=TYPES[t])

    def biased(n):
        return 0.1 * torch.randn(n, device="cuda", generator=g) if case["bias"] else None

    if what == "round":
        rows, cols = case["rows"], case["cols"]
        lines, length = (cols, rows) if case["columns"] else (rows, cols)
        s["x"] = _frames(g, rows, cols, case["pad"], kind, 1.0)
        s["codes"] = torch.empty(lines, -(-length // 128) * 128, device="cuda", dtype=torch.uint8)
        s["scales"] = torch.empty(lines, device="cuda")
        s["values"] = empty(rows, cols, kind)
        return s
    M, N, K = case["M"], case["N"], case["K"]
    s["x"] = _frames(g, M, K, case["pad"], kind, 1.0)
    # one workspace for all of a program's layers
    most = 4 * M * K + 8 * N * K + (8 * M * N + 4 * M * K if what == "gated_backward" else 0)
    s["ws"] = torch.empty(most + 2048 * (M + N + K) + (128 << 20), device="cuda", dtype=torch.uint8)
    if what == "linear":
        s["w"] = _weights_i8(g, N, K)
        s["bias"] = biased(N)
        s["y"] = empty(M, N, case["out"])
        return s
    if what == "gated_i8":
        s["wg"], s["wu"] = _weights_i8(g, N, K), _weights_i8(g, N, K)
    else:
        s["wg"], s["wu"] = _weights(g, N, K, case["weights"]), _weights(g, N, K, case["weights"])
    if what == "gated_backward":
        p, u = torch.randn(M, N, device="cuda", generator=g), torch.randn(M, N, device="cuda", generator=g)
        value, slope = _gate(p, case["gate"])       # what the forward pass kept
        s["slope_g"], s["slope_u"] = (u * slope).to(torch.bfloat16), value.to(torch.bfloat16)
        s["dh"] = _frames(g, M, N, case["pad"], kind, 1e-2)
        s["dx"] = empty(M, K, case["out"])
        s["dwg"], s["dwu"] = torch.empty(N, K, device="cuda"), torch.empty(N, K, device="cuda")
        s["dbg"], s["dbu"] = (torch.empty(N, device="cuda"), torch.empty(N, device="cuda")) if case["bias"] else (None, None)
        return s
    s["bg"], s["bu"] = biased(N), biased(N)
    s["h"] = empty(M, N, case["out"])
    keep = what == "gated" and case["keep"]
    s["slope_g"], s["slope_u"] = (empty(M, N, "bf16"), empty(M, N, "bf16")) if keep else (None, None)
    return s


# ---- the operators -------------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2205_03494_amd import omc
    what, case = s["what"], s["case"]
    if what == "round":
        omc.omc_i8_quantize(s["x"], s["codes"], s["scales"], by_columns=case["columns"], values=s["values"])
        return {"values": s["values"], "scales": s["scales"]}
    if what == "linear":
        omc.omc_i8_linear(s["x"], *s["w"], s["bias"], s["y"], s["ws"])
        return {"y": s["y"]}
    gate = {"sigmoid": omc.OMC_GATE_SIGMOID, "swish": omc.OMC_GATE_SWISH, "gelu": omc.OMC_GATE_GELU}[case["gate"]]
    if what == "gated_i8":
        omc.omc_i8_gated_linear(s["x"], *s["wg"], *s["wu"], s["bg"], s["bu"], gate, s["h"], s["ws"])
        return {"h": s["h"]}
    if what == "gated":
        omc.omc_gated_linear(s["x"], s["wg"], s["wu"], s["bg"], s["bu"], gate, s["h"], s["slope_g"], s["slope_u"], s["ws"])
        return {"h": s["h"], "slope_g": s["slope_g"], "slope_u": s["slope_u"]}
    omc.omc_gated_linear_backward(s["dh"], s["slope_g"], s["slope_u"], s["x"], s["wg"], s["wu"], s["dx"], s["dwg"], s["dwu"], s["dbg"], s["dbu"], s["ws"])
    return {"dx": s["dx"], "dwg": s["dwg"], "dwu": s["dwu"], "dbg": s["dbg"], "dbu": s["dbu"]}


def _gate(g, kind):
    """The gate's value and slope, in g's precision."""
    if kind == "gelu":
        below = 0.5 * torch.special.erfc(g * -math.sqrt(0.5))
        return g * below, below + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    s = 1.0 / (1.0 + torch.exp(-g))
    return (s, s * (1.0 - s)) if kind == "sigmoid" else (g * s, s * (1.0 + g * (1.0 - s)))


def _round(x, along):
    """Whole numbers nearest to x over its rows' (along = 1) or columns' (0) scales, and the scales."""
    scales = x.abs().amax(along, keepdim=True) / 127.0
    codes = torch.round(x.double() / torch.where(scales > 0, scales, 1.0).double())    # in 64 bits: ties are ties
    return codes.float(), scales


def _half(x):
    return x.to(torch.bfloat16).float()


def _run_plain(s):
    what, case = s["what"], s["case"]
    x = s["x"].float()
    if what == "round":
        codes, scales = _round(x, 0 if case["columns"] else 1)
        return {"values": (codes * scales).to(s["values"].dtype), "scales": scales.flatten()}
    if what in ("linear", "gated_i8"):
        codes, scales = _round(x, 1)

        def product(weights, bias):
            y = codes @ weights[0].view(torch.int8)[:, :x.shape[1]].float().t() * scales * weights[1]
            return y if bias is None else y + bias
        if what == "linear":
            return {"y": product(s["w"], s["bias"]).to(s["y"].dtype)}
        return {"h": (_gate(product(s["wg"], s["bg"]), case["gate"])[0] * product(s["wu"], s["bu"])).to(s["h"].dtype)}
    x, wg, wu = _half(x), _half(s["wg"]), _half(s["wu"])
    if what == "gated":
        g, u = x @ wg.t(), x @ wu.t()
        if case["bias"]:
            g, u = g + s["bg"], u + s["bu"]
        value, slope = _gate(g, case["gate"])
        kept = ((u * slope).to(torch.bfloat16), value.to(torch.bfloat16)) if case["keep"] else (None, None)
        return {"h": (value * u).to(s["h"].dtype), "slope_g": kept[0], "slope_u": kept[1]}
    dh = s["dh"].float()
    dg, du = dh * s["slope_g"].float(), dh * s["slope_u"].float()
    sums = (dg.sum(0), du.sum(0)) if case["bias"] else (None, None)
    dg, du = _half(dg), _half(du)
    return {"dx": (dg @ wg + du @ wu).to(s["dx"].dtype), "dwg": dg.t() @ x, "dwu": du.t() @ x, "dbg": sums[0], "dbu": sums[1]}


# ---- the same from the definition in 64 bits -----------------------------------------------------------------------

def _exact_codes(x, along):
    """Whole numbers by the distance to the one below: half belongs to the even one."""
    x = x.double()
    scales = (x.abs().max(along, keepdim=True).values / 127.0).float().double()
    t = x / torch.where(scales > 0, scales, 1.0)
    low = torch.floor(t)
    rest = t - low
    return low + ((rest > 0.5) | ((rest == 0.5) & (low % 2 != 0))).double(), scales


def _exact_gate(g, kind):
    if kind == "gelu":
        part = 0.5 * (1.0 - torch.erf(-g / math.sqrt(2.0)))
        return g * part, part + g / math.sqrt(2.0 * math.pi) * torch.exp(-g * g / 2.0)
    s = torch.sigmoid(g)
    rest = torch.sigmoid(-g)
    return (s, s * rest) if kind == "sigmoid" else (g * s, s + g * s * rest)


def exact(case, seed):
    s = prepare(case, seed)
    what = s["what"]
    if what == "round":
        codes, scales = _exact_codes(s["x"], 0 if case["columns"] else 1)
        return {"values": codes * scales, "scales": scales.reshape(-1)}
    if what in ("linear", "gated_i8"):
        codes, scales = _exact_codes(s["x"], 1)

        def product(weights, bias):
            w = weights[0].to(torch.int16)
            w = torch.where(w >= 128, w - 256, w)[:, :case["K"]].double() * weights[1].double()[:, None]
            y = (codes * scales) @ w.t()
            return y if bias is None else y + bias.double()
        if what == "linear":
            return {"y": product(s["w"], s["bias"])}
        return {"h": _exact_gate(product(s["wg"], s["bg"]), case["gate"])[0] * product(s["wu"], s["bu"])}
    x, wg, wu = (s[k].to(torch.bfloat16).double() for k in ("x", "wg", "wu"))
    if what == "gated":
        g, u = x @ wg.t(), x @ wu.t()
        if case["bias"]:
            g, u = g + s["bg"].double(), u + s["bu"].double()
        value, slope = _exact_gate(g, case["gate"])
        return {"h": value * u, "slope_g": slope * u if case["keep"] else None, "slope_u": value if case["keep"] else None}
    # (of dh in 32 bits the product is rounded to 32 bits first: a step of the definition)
    dh = s["dh"].double()
    dg, du = dh * s["slope_g"].double(), dh * s["slope_u"].double()
    dbg, dbu = (dg.sum(0), du.sum(0)) if case["bias"] else (None, None)
    dg, du = dg.float().to(torch.bfloat16).double(), du.float().to(torch.bfloat16).double()
    return {"dx": dg @ wg + du @ wu, "dwg": dg.t() @ x, "dwu": du.t() @ x, "dbg": dbg, "dbu": dbu}


def work(case):
    w = WIDTH[case["type"]]
    what = case["what"]
    if what == "round":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (2 * w + 1) + 4 * case["cols" if case["columns"] else "rows"], "flops": 4 * n}
    M, N, K = case["M"], case["N"], case["K"]
    v, sums = WIDTH[case["out"]], 4 * N * case["bias"]
    if what == "linear":
        return {"bytes": M * K * w + N * (K + 4) + M * N * v + sums, "flops": 2 * M * N * K}
    if what == "gated_i8":
        return {"bytes": M * K * w + 2 * N * (K + 4) + M * N * v + 2 * sums, "flops": 4 * M * N * K}
    layer = M * K * w + 2 * N * K * WIDTH[case["weights"]]
    if what == "gated":
        return {"bytes": layer + M * N * (v + 4 * case["keep"]) + 2 * sums, "flops": 4 * M * N * K}
    return {"bytes": layer + M * N * (w + 4) + M * K * v + 8 * N * K + 2 * sums, "flops": 8 * M * N * K}
