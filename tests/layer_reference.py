"""A layer with sparse weights in 64 bits on the CPU, from its formulas, and how far the kernels may be off.

Rounding to a type is off by at most u = eps / 2 of the value (and half of the smallest number that float16 holds).  A sum of n products in fp32, in
any order, is off by at most (n + 2) 2^-24 of the sum of the products' magnitudes.  The activations are z times a factor whose error is at most 2^-20: exp by a
product and a power of two, (1.5 |x| + 2) 2^-24 of its value, a reciprocal of one unit in the last place, erf of at most 16; |x| times the slope of the logistic function is below
0.23.  Their slopes are below 1.13, and off by at most 2^-19: two such factors and their sum."""
import math

import numpy as np
import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
SLOPE = 1.13
F32 = 2.0 ** -24

_erf = np.vectorize(math.erf, otypes=[np.float64])


def _logistic(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def activate(name, z):
    if name == "relu":
        return np.maximum(z, 0.0)
    if name == "silu":
        return z * _logistic(z)
    if name == "gelu":
        return 0.5 * z * (1.0 + _erf(z / math.sqrt(2.0)))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def slope(name, z):
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "silu":
        return _logistic(z) * (1.0 + z * _logistic(-z))
    if name == "gelu":
        return 0.5 * (1.0 + _erf(z / math.sqrt(2.0))) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if name == "gelu_tanh":
        a = math.sqrt(2.0 / math.pi)
        t = np.tanh(a * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * a * (1.0 + 3 * 0.044715 * z * z)
    return np.ones_like(z)


# ("heavy": 64 rows almost full, the others with as many entries as the density says)
# Products and gradients of sizes at which every kernel that the library chooses among runs: (m, k, N, density, kind, types), and a part of the name of the kernel (its launches are checked without a GPU, its results on one).
# Forward
KERNELS = [((4000, 4000, 4000, 0.05, "uniform", "f32 bf16 f16"), "layer_bandI{}Li4ELb0ELb1E"), ((6000, 6000, 6001, 0.02, "uniform", "f32 bf16 f16"), "layer_bandI{}Li4ELb0ELb0E"), ((6000, 6000, 6000, 0.01, "uniform", "f32"), "layer_bandI{}Li2"),
           ((9000, 9000, 9000, 0.0057, "zipf", "f32"), "layer_rows_allI{}"), ((6000, 6000, 6000, 0.02, "heavy", "f32 bf16 f16"), "layer_rows_allI{}"), ((6000, 6000, 5001, 0.02, "heavy", "f32 bf16 f16"), "layer_rows_allI{}"),
           ((4500, 4500, 2000, 0.003, "uniform", "bf16 f16"), "layer_rowsI{}Li32ELb0ELi8E"), ((4500, 4500, 2000, 0.008, "uniform", "bf16 f16"), "layer_rowsI{}Li32ELb0ELi16E"), ((5500, 5500, 2000, 0.006, "uniform", "bf16 f16"), "layer_rowsI{}Li16ELb0ELi16E"),
           ((4500, 4500, 2001, 0.003, "uniform", "bf16 f16"), "layer_rowsI{}Li16ELb1E"), ((6000, 6000, 500, 0.042, "uniform", "f32 bf16 f16"), "layer_realign"), ((6000, 6000, 301, 0.042, "uniform", "f32"), "layer_realign"), ((8000, 8000, 40, 0.002, "uniform", "bf16 f16"), "layer_rowsI{}Li8E"), ((8000, 8000, 21, 0.002, "uniform", "f32"), "layer_rowsI{}Li8E"),
           ((17000, 5000, 22, 0.002, "uniform", "bf16 f16"), "layer_rowsI{}Li4E"), ((5000, 5000, 1000, 0.004, "uniform", "bf16 f16"), "layer_rowsI{}Li16ELb0ELi8E"), ((3000, 9000, 300, 0.02, "zipf", "bf16 f16"), "layer_rowsI{}"),
           ((3000, 9000, 301, 0.02, "heavy", "f32 bf16 f16"), "layer_rowsI{}"),
           ((3000, 4000, 1, 0.2, "uniform", "f32 bf16 f16"), "layer_heldI{}Li64ELi1E"), ((3000, 3001, 2, 0.15, "loose", "f32 bf16 f16"), "layer_heldI{}Li64ELi2E"), ((3000, 3001, 3, 0.15, "loose", "f32 bf16 f16"), "layer_heldI{}Li64ELi4E"),
           ((3000, 3001, 31, 0.15, "loose", "bf16 f16"), "layer_heldI{}Li64ELi8E"), ((3000, 3001, 15, 0.15, "loose", "f32"), "layer_heldI{}Li64ELi4E"), ((600, 9900, 7, 0.1, "uniform", "bf16 f16"), "layer_heldI{}Li64ELi8E"),
           ((30000, 800, 2, 0.1, "loose", "f32 bf16 f16"), "layer_heldI{}Li16ELi2E"), ((40000, 700, 8, 0.02, "uniform", "bf16 f16"), "layer_heldI{}Li16ELi8E"), ((40000, 700, 7, 0.02, "uniform", "f32 bf16 f16"), "layer_heldI{}Li16E"),
           ((300, 30000, 6, 0.08, "uniform", "bf16 f16"), "layer_heldI{}Li64ELi2E"), ((300, 30000, 1, 0.05, "uniform", "f32"), "layer_heldI{}Li64ELi1E"), ((3000, 50000, 1, 0.005, "loose", "f32"), "layer_fewI{}Li64ELi1E"),
           ((3000, 50000, 3, 0.005, "loose", "f32 bf16 f16"), "layer_fewI{}Li64ELi4E"), ((3000, 90000, 7, 0.0001, "uniform", "bf16 f16"), "layer_fewI{}Li16ELi8E"), ((2000, 1900, 1001, 0.05, "uniform", "f32 bf16"), "layer_tileI{}"), ((2000, 1900, 1001, 0.05, "uniform", "f16"), "layer_tile_halves"), ((2000, 1000, 33, 0.25, "loose", "f16"), "layer_tile_halves"),
           ((1000, 2000, 100, 0.1, "heavy", "f16"), "layer_tile_halves"), ((2000, 1900, 20, 0.2, "uniform", "f32 bf16 f16"), "layer_tileI{}")]
# the gradient of the stored weights
VALUES_KERNELS = [((4000, 3900, 300, 0.2, "uniform", "bf16 f16"), "values_tilesI{}Li2ELi4ELi4"), ((3600, 4100, 513, 0.1, "loose", "bf16 f16"), "values_tilesI{}Li2ELi4ELi4"), ((1100, 1030, 1500, 0.4, "loose", "f32 bf16 f16"), "values_tilesI{}Li2ELi2ELi2"),
                  ((1000, 12000, 1500, 0.003, "uniform", "f32 bf16 f16"), "values_entriesI{}Li1E"), ((3000, 5000, 2001, 0.004, "zipf", "f32 bf16 f16"), "values_entriesI{}Li2E"), ((3000, 3000, 1200, 0.004, "zipf", "f32 bf16 f16"), "values_entriesI{}Li4E"),
                  ((9000, 3000, 24, 0.01, "loose", "f32 bf16 f16"), "values_"), ((3000, 3000, 1200, 0.008, "heavy", "f32 bf16 f16"), "values_entriesI{}Li4E"), ((6000, 6000, 500, 0.042, "uniform", "f32"), "layer_realign"), ((6000, 6000, 501, 0.042, "loose", "f32"), "layer_realign"), ((5000, 4000, 2001, 0.01, "uniform", "bf16 f16"), "layer_realign")]
MANGLED = {"f32": "f", "bf16": "DF16b", "f16": "DF16_"}


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def dense(m, k, row_ptr, cols, vals):
    """The weights and their magnitudes as dense matrices (entries that repeat add up)."""
    rows = np.repeat(np.arange(m), np.diff(row_ptr))
    W, M = np.zeros((m, k)), np.zeros((m, k))
    np.add.at(W, (rows, cols), vals.astype(np.float64))
    np.add.at(M, (rows, cols), np.abs(vals.astype(np.float64)))
    return W, M


def forward(W, M, lens, B, bias, act, residual, dtype):
    """((C, Z), how far each may be off); B, bias, residual as float64 arrays of what the kernel gets."""
    z, d = W @ B, M @ np.abs(B)
    off = (lens[:, None] + 2) * F32 * d
    if bias is not None:
        z = z + bias[:, None]
        off = off + F32 * np.abs(z)
    y = activate(act, z)
    off_y = SLOPE * off + (0.0 if act in ("none", "relu") else 2.0 ** -20 * (np.abs(z) + off))
    if residual is not None:
        y = y + residual
        off_y = off_y + F32 * np.abs(y)
    u, least = U[dtype], LEAST[dtype]
    return (y, z), (off_y + u * (np.abs(y) + off_y) + least, off + u * (np.abs(z) + off) + least)


def epilogue_grad(dC, Z, act, dtype):
    """((dZ, dbias), how far each may be off)"""
    g = dC if act == "none" else dC * slope(act, Z)
    off = np.zeros_like(g) if act in ("none", "relu") else 2.0 ** -19 * np.abs(dC)
    u, least = U[dtype], LEAST[dtype]
    n = dC.shape[1]
    return (g, g.sum(1)), (off + u * (np.abs(g) + off) + least, (off + (n + 1) * F32 * (np.abs(g) + off)).sum(1))


def grad_values(row_ptr, cols, dZ, B):
    rows = np.repeat(np.arange(len(row_ptr) - 1), np.diff(row_ptr))
    n = dZ.shape[1]
    return (dZ[rows] * B[cols]).sum(1), (n + 2) * F32 * (np.abs(dZ[rows]) * np.abs(B[cols])).sum(1)


def check(got, want, off, what=""):
    got = f64(got)
    assert got.shape == want.shape, what
    finite = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(got[~finite & ~np.isnan(want)], want[~finite & ~np.isnan(want)]), what
    bad = np.abs(got[finite] - want[finite]) > off[finite]
    assert not bad.any(), (what, int(bad.sum()), float((np.abs(got - want)[finite] / np.maximum(off[finite], 1e-300)).max()))


def check_on_gpu(got, want, off, what=""):
    """check() where both are on the GPU in 64 bits."""
    got = got.double()
    assert got.shape == want.shape, what
    bad = (got - want).abs() > off
    assert not bad.any() and torch.isfinite(got).all(), (what, int(bad.sum()), float(((got - want).abs() / off.clamp(min=1e-300)).max()))
