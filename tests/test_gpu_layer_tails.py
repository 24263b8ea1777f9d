"""The smooth activations and their slopes far to the left, where they themselves are small: against 64 bits relative to the value.

How far they may be off, u = 2^-24.  With x the exponent that an activation takes (silu z, gelu z^2 / 2, gelu_tanh 2 sqrt(2 / pi) (z + 0.044715 z^3)), the exponential and at most sixteen roundings around it are off by
16 u of the value.  An exponent formed in fp32 is off by as many u of itself as it has roundings, which the exponential turns into as many |x| u of its value: gelu_tanh has five (two of constants), gelu none in fp32, where
what the square loses is not left out, and one for the types of 2 bytes.  Those have an exponential of a product and a power of two, 1.5 |x| u more, and a polynomial for gelu that is off by 2^-22.  An exponential
below 2^-126, which is no normal number, may be 0: times z, that is up to 110, less than 2^-119 (and times z (2u)' = 244 where gelu_tanh's
exponent 2u comes to that, at z = -10.2, less than 2^-118).  A slope is a sum of two terms of either sign: the bound is of their magnitudes.  The rounding to the type comes on top."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2005_14469_amd import binding
from tests import layer_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
u = 2.0 ** -24
_erfc = np.vectorize(math.erfc, otypes=[np.float64])
A, B3 = math.sqrt(2.0 / math.pi), 0.044715


def logistic(x):
    e = np.exp(-np.abs(x))
    return np.where(x < 0, e, 1.0) / (1.0 + e)


def exponent(act, z):
    return {"silu": z, "gelu": 0.5 * z * z, "gelu_tanh": 2.0 * A * (z + B3 * z ** 3)}[act]


def value(act, z):
    return z * 0.5 * _erfc(-z / math.sqrt(2.0)) if act == "gelu" else z * logistic(exponent(act, z))


def slope(act, z):
    """The slope, and the sum of the magnitudes of its two terms."""
    if act == "gelu":
        a, b = 0.5 * _erfc(-z / math.sqrt(2.0)), z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    else:
        x = exponent(act, z)
        a, b = logistic(x), z * logistic(x) * logistic(-x) * (1.0 if act == "silu" else 2.0 * A * (1.0 + 3.0 * B3 * z * z))
    return a + b, a + np.abs(b)


def relative(act, z, T):
    x = np.abs(exponent(act, z))
    if T is torch.float32:
        return ({"silu": 0.0, "gelu": 0.0, "gelu_tanh": 5.0}[act] * x + 16.0) * u
    return ({"silu": 1.5, "gelu": 2.5, "gelu_tanh": 6.5}[act] * x + 16.0) * u + (2.0 ** -22 if act == "gelu" else 0.0)


def check(act, T, points, slopes=True):
    print(f"tails: {act} {T} {points[0]} .. {points[-1]}", flush=True)
    z = torch.from_numpy(points.astype(np.float32)).to(DEV).to(T)[None, :].contiguous()
    one = binding.gcoo_from_csr(1, 1, *[torch.from_numpy(a).to(DEV) for a in (np.array([0, 1], np.int32), np.zeros(1, np.int32), np.ones(1, np.float32))], 32, known_nnz=True)
    z64, U, least = ref.f64(z), ref.U[T], ref.LEAST[T] + 2.0 ** -119
    rel = relative(act, z64, T)
    want = value(act, z64)
    ref.check(binding.gcoo_spdm_epilogue(one, z, activation=act), want, (rel + U * (1.0 + rel)) * np.abs(want) + least, "value")
    if not slopes:
        return
    want, both = slope(act, z64)
    ref.check(binding.gcoo_epilogue_grad(torch.ones_like(z), Z=z, activation=act)[0], want, rel * both + U * (np.abs(want) + rel * both) + least + 2.0 ** -119, "slope")


GRID = np.linspace(-12.0, 12.0, 4801)


def test_gelu_in_32_bits():
    """Phi(z) as 1 + erf would have lost every bit at z = -5.5, where gelu is -1e-7."""
    check("gelu", torch.float32, GRID)
    check("gelu", torch.float32, np.linspace(-13.0, -1.0, 50001))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_gelu_in_16_bits(dtype):
    check("gelu", TYPES[dtype], GRID)


def test_silu_and_gelu_tanh_in_32_bits():
    check("silu", torch.float32, np.linspace(-80.0, 80.0, 40001), slopes=False)
    check("gelu_tanh", torch.float32, GRID, slopes=False)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_gates_far_out(act, dtype):
    """Where the exponential is far from 1, the slope is not what it is at some nearer z."""
    check(act, TYPES[dtype], np.concatenate([np.linspace(-110.0, -70.0, 801), GRID, np.linspace(70.0, 110.0, 801)]))


def test_slopes_of_gates_in_32_bits():
    check("silu", torch.float32, np.linspace(-80.0, 80.0, 40001))
    check("gelu_tanh", torch.float32, GRID)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_of_infinite_sums(dtype):
    """As the formulas have it: infinite on the right, -infinity times 0 on the left but for relu; very large finite sums give 0 there."""
    big = 60000.0 if dtype == "f16" else 3e38
    z = torch.tensor([[-math.inf, -big, big, math.inf, math.nan]], device=DEV, dtype=TYPES[dtype])
    one = binding.gcoo_from_csr(1, 1, *[torch.from_numpy(a).to(DEV) for a in (np.array([0, 1], np.int32), np.zeros(1, np.int32), np.ones(1, np.float32))], 32, known_nnz=True)
    for act in ("relu", "silu", "gelu", "gelu_tanh"):
        y = binding.gcoo_spdm_epilogue(one, z, activation=act)[0]
        assert torch.isnan(y[4]) and torch.equal(y[1:4], torch.stack([torch.zeros_like(z[0, 0]), z[0, 2], z[0, 3]])), (act, y)
        assert y[0] == 0 if act == "relu" else torch.isnan(y[0]), (act, y)
