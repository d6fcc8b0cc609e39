"""Plain 64-bit references of the layer's operators, on the CPU, written from the definitions (numpy)."""
import ctypes as C

import numpy as np
import torch

from paper_2205_03494_amd import omc

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def padded(n):
    return -(-n // 128) * 128


def quantize(x):
    """(codes [rows, padded / 2], scales [rows, padded / 32], values [rows, cols] in fp64) of a float array, blocked along its rows."""
    rows, cols = x.shape
    x = np.asarray(x, dtype=np.float64)
    wide = np.zeros((rows, padded(cols)))
    wide[:, :cols] = x
    b = wide.reshape(rows, -1, 32)
    bad = ~np.isfinite(b).all(-1)
    b = np.where(bad[..., None], 0.0, b)
    top = np.abs(b).max(-1)
    e = np.where(top > 0, np.frexp(top)[1] - 1 - 2, -127)
    e = np.maximum(e, -127)
    u = np.ldexp(np.abs(b), -e[..., None])
    assert (u < 8).all()
    code = np.zeros(u.shape, np.int64)
    best = np.full(u.shape, np.inf)
    for k in (0, 2, 4, 6, 1, 3, 5, 7):       # of two equally near the even one, which is looked at first
        d = np.abs(u - GRID[k])
        code = np.where(d < best, k, code)
        best = np.minimum(d, best)
    value = np.ldexp(GRID[code], e[..., None]) * np.where(np.signbit(b), -1.0, 1.0)
    value[bad] = np.nan
    code = np.where(np.signbit(b), code + 8, code)
    code[bad] = 0
    scale = np.where(bad, 255, e + 127).astype(np.uint8)
    flat = code.reshape(rows, -1).astype(np.uint8)
    return flat[:, 0::2] | (flat[:, 1::2] << 4), scale, value.reshape(rows, -1)[:, :cols]


def values(codes, scales, cols):
    """fp64 values of codes and scales."""
    c = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], -1).astype(np.int64)
    v = GRID[c & 7] * np.where(c & 8, -1.0, 1.0)
    unit = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (v * np.repeat(unit, 32, 1))[:, :cols]


def layer_norm(x, gamma, beta, eps):
    mean = x.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    return (x - mean) * rstd * gamma + beta, mean[:, 0], rstd[:, 0]


def layer_norm_backward(dy, x, gamma, mean, rstd):
    hat = (x - mean[:, None]) * rstd[:, None]
    u = dy * gamma
    dx = rstd[:, None] * (u - u.mean(1, keepdims=True) - hat * (u * hat).mean(1, keepdims=True))
    return dx, (dy * hat).sum(0), dy.sum(0)


def product_bound(a, b, K):
    """How far fp32 sums may be from a b^T: K / 128 instructions one after the other, parts joined, two bits of an instruction's own sum."""
    return product_bound_of(np.abs(a) @ np.abs(b).T, K)


def product_bound_of(magnitudes, K):
    return (K / 128 + 16) * 2.0 ** -23 * magnitudes


def rounding(ref, dtype):
    return np.abs(ref) * (2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -23)


def as64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def product_tile(M, N, K):
    """(index of the tile that the product takes, is its contraction cut, more tiles than the chip holds at a time): 256 x 256, 128 x 128, 64 x 64."""
    fn = omc._lib.omc_internal_mx4_tile
    fn.restype, fn.argtypes = C.c_int, [C.c_uint32] * 3
    tile, parts = fn(M, N, K) % 16, fn(M, N, K) // 16
    bm, bn, at_a_time = ((256, 256, 256), (128, 128, 256), (64, 64, 512))[tile]
    return tile, parts > 1, -(-M // bm) * -(-N // bn) * parts > at_a_time


def pair_tile(M, N, K):
    """Index of the tile in which both products of a backward pass go together; -1: each in a launch of its own."""
    fn = omc._lib.omc_internal_mx4_pair_tile
    fn.restype, fn.argtypes = C.c_int, [C.c_uint32] * 3
    return fn(M, N, K)


# Products that between them take every tile, with fewer and with more of them than the chip holds at a time, whole and odd numbers of 128s, and contractions in parts.
PRODUCTS = [(7242, 1702, 3983), (2213, 5436, 3864), (7859, 3827, 3283), (3814, 7658, 3103), (1069, 4825, 131), (653, 7529, 33), (2457, 3302, 130),
            (4624, 1681, 34), (70, 8513, 8934), (69, 8432, 8525), (512, 512, 65536), (8366, 138, 132), (8356, 131, 33), (406, 8690, 133),
            (531, 6706, 33), (36, 34, 129), (257, 6724, 461), (282, 6605, 289), (34, 37, 3758), (33, 35, 3698), (1798, 8103, 43), (4013, 7311, 1304),
            (644, 8567, 35), (2931, 1062, 320), (471, 6654, 1532), (332, 648, 25899), (641, 359, 26001), (34, 33, 5207), (37, 37, 4868),
            (260, 150, 9001)]

# Results of 32 MB and more in bf16, whose rows are whole cache lines, in every tile; whole tiles and not.
LARGE_RESULTS = [(8192, 2048, 300), (8190, 2112, 1000), (4097, 4096, 300), (262145, 64, 40)]

# Backward passes: few rows in either product, both together in either tile, apart.
BACKWARD = [(1, 1, 1, 0), (1, 64, 96, 0), (3, 33, 65, 1), (40, 96, 300, 0), (128, 64, 64, 0), (129, 257, 130, 3), (300, 520, 70, 0), (1003, 243, 97, 1),
            (2100, 128, 384, 0), (257, 65, 700, 1), (4001, 600, 1500, 0), (140001, 33, 40, 0), (2990, 1100, 1555, 1), (2048, 8192, 2304, 0),
            (20000, 1, 20, 0), (50001, 33, 20, 1)]
