"""The sixteen-wave product and the launch of uneven rows with every form of the epilogue: C as the residual, nothing but C, each activation; against dense products in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2005_14469_amd import binding
from tests import layer_reference as ref
from tests.test_gpu_layer import DEV, TYPES, csr, matrix

pytestmark = pytest.mark.gpu

# the sizes of layer_reference.KERNELS that these kernels are launched for (which is checked without a GPU)
SHAPES = [(*shape[:5], dtype) for shape, name in ref.KERNELS if name.startswith(("layer_bandI", "layer_rows_allI")) for dtype in shape[5].split()]
# activation, bias, residual ("C": C itself), Z
FORMS = [("none", False, None, False), ("gelu", False, "C", False), ("silu", True, "C", True), ("gelu_tanh", True, "another", False), ("relu", False, None, True), ("none", True, "C", False)]


def activate(act, z):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z * torch.special.expit(z)
    if act == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    if act == "gelu_tanh":
        return z * torch.special.expit(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
    return z


def test_there_are_such_sizes():
    assert len(SHAPES) >= 14 and {s[5] for s in SHAPES} == set(TYPES)


@pytest.mark.parametrize("m,k,N,density,kind,dtype", SHAPES)
def test_every_form_of_the_epilogue(m, k, N, density, kind, dtype):
    """Off by what layer_reference.forward() allows: n + 2 roundings of the sum of the magnitudes, the bias's, 1.13 times that behind an activation and 2^-20 |z| for it, the residual's, the type's."""
    T = TYPES[dtype]
    arrays = csr(m, k, density, m + N, kind)
    A = matrix(m, k, arrays)
    lens = torch.from_numpy(np.diff(arrays[0])).to(DEV)
    at = torch.repeat_interleave(torch.arange(m, device=DEV), lens), torch.from_numpy(arrays[1]).to(DEV).long()
    vals = torch.from_numpy(arrays[2]).to(DEV).double()
    gen = torch.Generator(device=DEV)
    gen.manual_seed(m + k)
    # (values such that z is of order one: the activations bend there)
    B, R = (0.3 * torch.randn((k, N), generator=gen, device=DEV)).to(T), torch.randn((m, N), generator=gen, device=DEV).to(T)
    b = torch.randn(m, generator=gen, device=DEV)
    W = torch.zeros((m, k), dtype=torch.float64, device=DEV).index_put_(at, vals, accumulate=True)
    product = W @ B.double()
    W.zero_().index_put_(at, vals.abs(), accumulate=True)
    sums = (lens.double()[:, None] + 2) * ref.F32 * (W @ B.double().abs())
    del W
    u, least = ref.U[T], ref.LEAST[T]
    for act, bias, residual, keep in FORMS:
        print(f"band: {m} x {k} x {N} {density} {kind} {dtype} {act} bias={bias} residual={residual} Z={keep}", flush=True)
        C = torch.full((m, N + 3), 7.0, dtype=T, device=DEV)
        if residual == "C":
            C[:, :N] = R
        Z = torch.full((m, N + 1), 7.0, dtype=T, device=DEV) if keep else None
        binding.gcoo_spdm_epilogue(A, B, bias=b if bias else None, activation=act, residual={None: None, "C": C[:, :N], "another": R}[residual], C_out=C[:, :N], Z_out=Z[:, :N] if keep else None)
        z, off = product, sums
        if bias:
            z = z + b.double()[:, None]
            off = off + ref.F32 * z.abs()
        if keep:
            ref.check_on_gpu(Z[:, :N], z, off + u * (z.abs() + off) + least, "Z")
            assert torch.all(Z[:, N:] == 7.0)
        y = activate(act, z)
        off = off if act in ("none", "relu") else ref.SLOPE * off + 2.0 ** -20 * (z.abs() + off)
        if residual:
            y = y + R.double()
            off = off + ref.F32 * y.abs()
        ref.check_on_gpu(C[:, :N], y, off + u * (y.abs() + off) + least, "C")
        assert torch.all(C[:, N:] == 7.0)
        del z, y, off
