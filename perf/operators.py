"""A linear layer in 4-bit microscaled floats and the layer norm before it, as they are timed.

A feed-forward module of a Conformer takes y = norm(x), multiplies the 4-bit images of y and of its weights, and on the way
back forms both gradients of the product the same way, and the norm's.  The cases are single uses of these: one frame of a
stream, an ordinary batch of frames (8192 of them, layers of 1024 <-> 4096 as in the repository's benchmark), large and
ragged ones.

MX4: 32 neighbours along the contraction share a power of two, 2^e with e = max(floor(log2(largest magnitude)) - 2, -127),
and hold an E2M1 value each (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives; nearest, ties to even, saturating).  A row is padded
to a multiple of 128 values; two codes a byte, the first in the low four bits; the power as a byte e + 127.
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
WIDTH = {"f32": 4, "bf16": 2}
MOST_NORM = 32768 * 4096
MOST_ROUND = 16384 * 8192
MOST_LINEAR = 16384 * 8192 * 8192
MOST_BACKWARD = 8192 * 4096 * 4096


def listed():
    return [
        # one frame of a streaming encoder: latency of a call
        {"name": "norm_frame", "what": "norm", "rows": 1, "cols": 512, "pad": 0, "type": "bf16", "out": "bf16"},
        # a batch's frames before a feed-forward module, residual stream in 32 bits, the product's input in 16
        {"name": "norm_batch", "what": "norm", "rows": 8192, "cols": 1024, "pad": 0, "type": "f32", "out": "bf16"},
        # a short batch, width and stride no multiple of anything: a slice of a wider buffer
        {"name": "norm_grad_ragged", "what": "norm_backward", "rows": 1237, "cols": 971, "pad": 3, "type": "f32", "out": "f32"},
        # a long batch of a wide model
        {"name": "norm_grad_large", "what": "norm_backward", "rows": 32768, "cols": 4096, "pad": 0, "type": "bf16", "out": "bf16"},
        # weights as quantisation-aware training sees them: a matrix of odd sizes
        {"name": "round_ragged", "what": "round", "rows": 971, "cols": 243, "pad": 0, "type": "f32"},
        # all of a large batch's activations
        {"name": "round_large", "what": "round", "rows": 16384, "cols": 8192, "pad": 0, "type": "bf16"},
        # one frame through a feed-forward layer's 4-bit weights
        {"name": "linear_frame", "what": "linear", "M": 1, "N": 4096, "K": 1024, "pad": 0, "type": "bf16", "out": "bf16", "bias": True},
        # some streams served together, wide layer, sizes off the tiles
        {"name": "linear_streams", "what": "linear", "M": 29, "N": 8200, "K": 8192, "pad": 0, "type": "bf16", "out": "f32", "bias": False},
        # an ordinary batch through the same layer
        {"name": "linear_batch", "what": "linear", "M": 8192, "N": 4096, "K": 1024, "pad": 0, "type": "bf16", "out": "bf16", "bias": True},
        # the largest product
        {"name": "linear_large", "what": "linear", "M": 16384, "N": 8192, "K": 8192, "pad": 0, "type": "bf16", "out": "bf16", "bias": False},
        # backward through a small layer, ragged batch
        {"name": "linear_grad_ragged", "what": "linear_backward", "M": 1003, "N": 971, "K": 243, "pad": 1, "type": "f32", "out": "f32", "bias": True},
        # backward through the layer behind it, ordinary batch
        {"name": "linear_grad_batch", "what": "linear_backward", "M": 8192, "N": 1024, "K": 4096, "pad": 0, "type": "bf16", "out": "bf16", "bias": True},
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Any size between the listed ones' least and most; half of the widths are whole blocks of 32, a quarter of the inputs slices."""
    what = rng.choice(("norm", "norm_backward", "round", "linear", "linear", "linear", "linear_backward", "linear_backward"))
    while True:
        def wide(lo, hi):
            n = _between(rng, lo, hi)
            return max(32, n // 32 * 32) if rng.random() < 0.5 else n
        case = {"what": what, "pad": rng.randint(1, 64) if rng.random() < 0.25 else 0, "type": rng.choice(("bf16", "bf16", "f32"))}
        if what in ("norm", "norm_backward"):
            case |= {"rows": _between(rng, 1, 32768), "cols": wide(64, 8192), "out": rng.choice(("bf16", case["type"]))}
            size, most = case["rows"] * case["cols"] * WIDTH[case["type"]], MOST_NORM * 2
        elif what == "round":
            case |= {"rows": _between(rng, 1, 16384), "cols": wide(32, 8192)}
            size, most = case["rows"] * case["cols"] * WIDTH[case["type"]], MOST_ROUND * 2
        else:
            forward = what == "linear"
            case |= {"M": _between(rng, 1, 16384 if forward else 8192), "N": wide(64, 8192 if forward else 4096), "K": wide(64, 8192 if forward else 4096),
                     "out": rng.choice(("bf16", "f32")), "bias": rng.random() < 0.5}
            size, most = case["M"] * case["N"] * case["K"], MOST_LINEAR if forward else MOST_BACKWARD
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


def _weights(g, rows, cols):
    """A weight matrix's codes and scales, its rows' blocks along `cols`, in the layout that the products take."""
    wide = -(-cols // 128) * 128
    w = torch.zeros(rows, wide, device="cuda")
    w[:, :cols] = torch.randn(rows, cols, device="cuda", generator=g) / math.sqrt(cols)
    w = w.view(rows, wide // 32, 32)
    e = _exponents(w)
    k = _steps(w.abs() * _power(-e))
    k = (k + torch.where(w < 0, 8, 0)).to(torch.uint8).view(rows, wide // 2, 2)
    return (k[..., 0] | (k[..., 1] << 4)).contiguous(), (e + 127).to(torch.uint8).view(rows, wide // 32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    what, kind = case["what"], case["type"]
    s = {"case": case, "what": what}

    def empty(rows, cols, t):
        return torch.empty(rows, cols, device="cuda", dtype=TYPES[t])

    if what in ("norm", "norm_backward"):
        rows, cols = case["rows"], case["cols"]
        s["x"] = _frames(g, rows, cols, case["pad"], kind, 1.0)
        s["gamma"] = 1.0 + 0.1 * torch.randn(cols, device="cuda", generator=g)
        s["beta"] = 0.1 * torch.randn(cols, device="cuda", generator=g)
        s["mean"], s["rstd"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        if what == "norm":
            s["y"] = empty(rows, cols, case["out"])
        else:
            for i in range(0, rows, 4096):     # what the forward pass kept
                part = s["x"][i:i + 4096].double()
                s["mean"][i:i + 4096] = part.mean(1)
                s["rstd"][i:i + 4096] = (part.var(1, correction=0) + EPS).rsqrt()
            s["dy"] = _frames(g, rows, cols, case["pad"], case["out"], 1e-2)
            s["dx"], s["dgamma"], s["dbeta"] = empty(rows, cols, kind), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
            s["ws"] = torch.empty(16384 * cols + (1 << 20), device="cuda", dtype=torch.uint8)
    elif what == "round":
        rows, cols = case["rows"], case["cols"]
        wide = -(-cols // 128) * 128
        s["x"] = _frames(g, rows, cols, case["pad"], kind, 1.0)
        s["codes"] = torch.empty(rows, wide // 2, device="cuda", dtype=torch.uint8)
        s["scales"] = torch.empty(rows, wide // 32, device="cuda", dtype=torch.uint8)
        s["values"] = empty(rows, cols, kind)
    else:
        M, N, K = case["M"], case["N"], case["K"]
        s["x"] = _frames(g, M, K, case["pad"], kind, 1.0)
        # one workspace for all of a program's layers
        s["ws"] = torch.empty(2 * (M * K + M * N) + 16 * (M + N + K) * 128 + (64 << 20), device="cuda", dtype=torch.uint8)
        if what == "linear":
            s["codes"], s["scales"] = _weights(g, N, K)
            s["bias"] = 0.1 * torch.randn(N, device="cuda", generator=g) if case["bias"] else None
            s["y"] = empty(M, N, case["out"])
        else:
            s["codes"], s["scales"] = _weights(g, K, N)
            s["dy"] = _frames(g, M, N, case["pad"], kind, 1e-2)
            s["dx"], s["dw"] = empty(M, K, case["out"]), torch.empty(K, N, device="cuda")
            s["dbias"] = torch.empty(N, device="cuda") if case["bias"] else None
    return s


# ---- the operators -------------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2205_03494_amd import omc
    what = s["what"]
    if what == "norm":
        omc.omc_layer_norm(s["x"], s["gamma"], s["beta"], EPS, s["y"], s["mean"], s["rstd"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if what == "norm_backward":
        omc.omc_layer_norm_backward(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"], s["ws"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if what == "round":
        omc.omc_mx4_quantize(s["x"], s["codes"], s["scales"], values=s["values"])
        return {"values": s["values"]}
    if what == "linear":
        omc.omc_mx4_linear(s["x"], s["codes"], s["scales"], s["bias"], s["y"], s["ws"])
        return {"y": s["y"]}
    omc.omc_mx4_linear_backward(s["dy"], s["x"], s["codes"], s["scales"], s["dx"], s["dw"], s["dbias"], s["ws"])
    return {"dx": s["dx"], "dw": s["dw"], "dbias": s["dbias"]}


def _power(e):
    """2^e in fp32 for whole e of -127 .. 127 (2^-127 has no exponent field of its own)."""
    bits = torch.where(e == -127, 1 << 22, (e + 127) << 23)
    return bits.to(torch.int32).view(torch.float32)


def _exponents(blocks):
    a = blocks.abs().amax(-1, keepdim=True)
    e = torch.frexp(a)[1] - 3
    return torch.where(a > 0, e.clamp(min=-127), -127)


def _steps(v):
    """Index of the E2M1 magnitude nearest to v in [0, 8): 0 .. 7, ties to the even index."""
    fine, middle, coarse = torch.round(v * 2), torch.round(v) + 2, torch.round(v * 0.5) + 4
    return torch.where(v < 2, fine, torch.where(v < 4, middle, coarse)).clamp(max=7)


def _table():
    return torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")


def _round(x):
    """MX4 values of a matrix in fp32, blocks along its rows; padded to whole blocks."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % 32)).view(rows, -1, 32)
    e = _exponents(x)
    k = _steps(x.abs() * _power(-e))
    return (torch.copysign(_table()[k.to(torch.int64)], x) * _power(e)).view(rows, -1)[:, :cols]


def _decoded(codes, scales, cols):
    k = torch.stack((codes & 15, codes >> 4), -1).to(torch.int64).view(codes.shape[0], -1, 32)
    table = torch.cat((_table(), -_table()))
    return (table[k] * _power(scales.to(torch.int32) - 127).unsqueeze(-1)).view(codes.shape[0], -1)[:, :cols]


def _run_plain(s):
    what = s["what"]
    x = s["x"].float()
    if what == "norm":
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
        return {"y": (d * rstd * s["gamma"] + s["beta"]).to(s["y"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if what == "norm_backward":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        hat = (x - s["mean"][:, None]) * rstd
        u = dy * s["gamma"]
        dx = rstd * (u - u.mean(1, keepdim=True) - hat * (u * hat).mean(1, keepdim=True))
        return {"dx": dx.to(s["dx"].dtype), "dgamma": (dy * hat).sum(0), "dbeta": dy.sum(0)}
    if what == "round":
        return {"values": _round(x).to(s["values"].dtype)}
    if what == "linear":
        y = _round(x) @ _decoded(s["codes"], s["scales"], x.shape[1]).t()
        return {"y": (y if s["bias"] is None else y + s["bias"]).to(s["y"].dtype)}
    dy = s["dy"].float()
    dx = _round(dy) @ _decoded(s["codes"], s["scales"], dy.shape[1]).t()
    dw = _round(x.t().contiguous()) @ _round(dy.t().contiguous()).t()
    return {"dx": dx.to(s["dx"].dtype), "dw": dw, "dbias": None if s["dbias"] is None else dy.sum(0)}


# ---- the same from the definition in 64 bits -----------------------------------------------------------------------

def _exact_round(x):
    """Every value's nearest neighbour by the midpoints between E2M1 values: a tie belongs to the even one of the two."""
    rows, cols = x.shape
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda", dtype=torch.float64)
    mids = (grid[1:] + grid[:-1]) / 2
    below = torch.nextafter(mids, torch.zeros_like(mids))
    mids[1::2] = below[1::2]           # between an odd and the next even value: the tie goes up
    b = torch.nn.functional.pad(x.double(), (0, -cols % 32)).reshape(rows, -1, 32)
    top = b.abs().max(-1, keepdim=True).values
    whole = torch.floor(torch.log2(torch.where(top > 0, top, 1.0)))
    unit = torch.exp2(torch.clamp(torch.where(top > 0, whole, -125.0) - 2.0, min=-127.0))
    unit = torch.where(top / unit >= 8.0, unit * 2.0, torch.where((top / unit < 4.0) & (unit > 2.0 ** -127), unit / 2.0, unit))
    near = torch.bucketize((b.abs() / unit).contiguous(), mids)
    return (torch.sign(b) * grid[near] * unit).reshape(rows, -1)[:, :cols]


def _exact_weights(codes, scales, cols):
    c = codes.to(torch.int64)
    c = torch.stack((c % 16, c // 16), 2).reshape(c.shape[0], -1)
    half = (c % 8).double()
    size = torch.where(half < 4, half / 2, torch.where(half < 6, half - 2, 2 * half - 8))
    unit = torch.exp2(scales.double() - 127.0).repeat_interleave(32, 1)
    return (torch.where(c >= 8, -size, size) * unit)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    what = s["what"]
    if what == "norm":
        y = torch.empty(s["y"].shape, device="cuda", dtype=torch.float64)
        mean, rstd = torch.empty(len(y), device="cuda", dtype=torch.float64), torch.empty(len(y), device="cuda", dtype=torch.float64)
        for i in range(0, len(y), 4096):
            x = s["x"][i:i + 4096].double()
            mean[i:i + 4096] = x.mean(1)
            x -= mean[i:i + 4096, None]
            rstd[i:i + 4096] = (x.square().mean(1) + EPS).pow(-0.5)
            y[i:i + 4096] = x * rstd[i:i + 4096, None] * s["gamma"].double() + s["beta"].double()
        return {"y": y, "mean": mean, "rstd": rstd}
    if what == "norm_backward":
        dx = torch.empty(s["dx"].shape, device="cuda", dtype=torch.float64)
        dgamma = torch.zeros(dx.shape[1], device="cuda", dtype=torch.float64)
        dbeta = torch.zeros_like(dgamma)
        for i in range(0, len(dx), 4096):
            x, dy, r = s["x"][i:i + 4096].double(), s["dy"][i:i + 4096].double(), s["rstd"][i:i + 4096].double()[:, None]
            hat = (x - s["mean"][i:i + 4096].double()[:, None]) * r
            dgamma += (dy * hat).sum(0)
            dbeta += dy.sum(0)
            dy = dy * s["gamma"].double()
            dx[i:i + 4096] = (dy - (dy.sum(1, keepdim=True) + hat * (dy * hat).sum(1, keepdim=True)) / dx.shape[1]) * r
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if what == "round":
        return {"values": _exact_round(s["x"])}
    if what == "linear":
        y = _exact_round(s["x"]) @ _exact_weights(s["codes"], s["scales"], case["K"]).t()
        return {"y": y if s["bias"] is None else y + s["bias"].double()}
    dw = _exact_round(s["x"].t().contiguous()) @ _exact_round(s["dy"].t().contiguous()).t()
    dx = _exact_round(s["dy"]) @ _exact_weights(s["codes"], s["scales"], case["N"]).t()
    return {"dx": dx, "dw": dw, "dbias": None if s["dbias"] is None else s["dy"].double().sum(0)}


def work(case):
    w = WIDTH[case["type"]]
    what = case["what"]
    if what in ("norm", "norm_backward"):
        rows, cols, v = case["rows"], case["cols"], WIDTH[case["out"]]
        if what == "norm":
            return {"bytes": rows * cols * (w + v) + 8 * rows + 8 * cols, "flops": 8 * rows * cols}
        return {"bytes": rows * cols * (2 * w + v) + 8 * rows + 12 * cols, "flops": 14 * rows * cols}
    if what == "round":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (2 * w + 17 / 32), "flops": 4 * n}
    M, N, K = case["M"], case["N"], case["K"]
    if what == "linear":
        return {"bytes": M * K * w + N * K * 17 / 32 + M * N * WIDTH[case["out"]] + 4 * N * case["bias"], "flops": 2 * M * N * K}
    return {"bytes": (M * K + M * N) * w + K * N * 17 / 32 + M * K * WIDTH[case["out"]] + 4 * K * N + 4 * N * case["bias"], "flops": 4 * M * N * K}
