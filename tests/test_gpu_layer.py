"""A layer with sparse weights - the product with its epilogue, its gradients, clipping - against the same in 64 bits (layer_reference.py)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2005_14469_amd import binding, workloads
from tests import layer_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def csr(m, k, density, seed, kind="uniform"):
    """row_ptr, cols, vals: "uniform", "zipf" (rows of very different lengths), "loose" (columns in no order, some twice, every third row empty),
    "heavy" (64 rows from row 700 on almost full)"""
    if kind == "zipf":
        w = workloads.zipf_rows(m, k, 1, seed, row_max=min(k, 3000))
        return w.row_ptr, w.col_idx, w.vals
    rng = np.random.default_rng(seed)
    if kind == "heavy":
        mask = rng.random((m, k), dtype=np.float32) < density
        mask[700:764] = rng.random((64, k), dtype=np.float32) < 0.9
        cells = np.flatnonzero(mask)
        return workloads.csr_from_cells(m, k, cells, rng.standard_normal(len(cells)).astype(np.float32))
    if kind == "uniform" and m * k > 4000000:
        cells = np.flatnonzero(rng.random((m, k), dtype=np.float32) < density)
        return workloads.csr_from_cells(m, k, cells, rng.standard_normal(len(cells)).astype(np.float32))
    w = workloads.uniform_random(m, k, 1, 1 - density, seed)
    if kind == "uniform":
        return w.row_ptr, w.col_idx, w.vals
    lens = rng.integers(0, max(2, int(2 * density * k)), size=m)
    lens[::3] = 0
    row_ptr = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    return row_ptr, rng.integers(0, k, size=row_ptr[-1]).astype(np.int32), rng.standard_normal(row_ptr[-1]).astype(np.float32)


def matrix(m, k, arrays, p=32):
    return binding.gcoo_from_csr(m, k, *[torch.from_numpy(x).to(DEV) for x in arrays], p, known_nnz=True)


class Padded:
    """A rows x N matrix inside a larger allocation of 7s, `shift` elements behind its beginning, rows `extra` elements apart; whole() that nothing else was written."""

    def __init__(self, rows, N, dtype, extra=0, shift=0, fill=None):
        self.all = torch.full((max(rows, 1) * (N + extra) + shift + 8,), 7.0, dtype=dtype, device=DEV)
        self.t = self.all[shift:shift + max(rows, 1) * (N + extra)].view(max(rows, 1), N + extra)[:rows, :N]
        self.rows, self.N, self.extra, self.shift = rows, N, extra, shift
        if fill is not None:
            self.t.copy_(fill)

    def whole(self):
        other = self.all.clone()
        other[self.shift:self.shift + max(self.rows, 1) * (self.N + self.extra)].view(max(self.rows, 1), self.N + self.extra)[:self.rows, :self.N] = 7.0
        return bool((other == 7.0).all())


def normal(rng, *shape, dtype=torch.float32):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DEV).to(dtype)


def forward_case(m, k, N, density, kind, dtype, act, bias, residual, keep, extra=0, shift=0, p=32, seed=None):
    seed = seed or m + 3 * k + 5 * N
    print(f"forward: {m} x {k} x {N} {density} {kind} {dtype} {act} bias={bias} residual={residual} keep={keep} extra={extra} shift={shift} p={p}", flush=True)
    arrays = csr(m, k, density, seed, kind)
    A = matrix(m, k, arrays, p)
    rng = np.random.default_rng(seed)
    B = Padded(k, N, dtype, extra, shift, normal(rng, k, N, dtype=dtype))
    R = Padded(m, N, dtype, extra, shift, normal(rng, m, N, dtype=dtype)) if residual else None
    b = normal(rng, m) if bias else None
    Cp, Zp = Padded(m, N, dtype, extra, shift), (Padded(m, N, dtype, extra, shift) if keep else None)
    got = binding.gcoo_spdm_epilogue(A, B.t, bias=b, activation=act, residual=R.t if R else None, C_out=Cp.t, Z_out=Zp.t if Zp else None)
    assert got is Cp.t
    torch.cuda.synchronize()
    W, M = ref.dense(m, k, *arrays)
    (y, z), (off_y, off_z) = ref.forward(W, M, np.diff(arrays[0]), ref.f64(B.t), ref.f64(b), act, ref.f64(R.t) if R else None, dtype)
    ref.check(Cp.t, y, off_y, "C")
    assert Cp.whole() and B.whole()
    if Zp:
        ref.check(Zp.t, z, off_z, "Z")
        assert Zp.whole()
    again = torch.empty_like(Cp.t)
    binding.gcoo_spdm_epilogue(A, B.t, bias=b, activation=act, residual=R.t if R else None, C_out=again)
    assert torch.equal(again, Cp.t)                                    # the same bits, with Z and without
    if R:
        inside = R.t.clone()
        binding.gcoo_spdm_epilogue(A, B.t, bias=b, activation=act, residual=inside, C_out=inside)
        assert torch.equal(inside, again)


SHAPES = [(1, 1, 1, 1.0, "uniform"), (1, 700, 1, 0.5, "uniform"), (70, 1, 9, 1.0, "uniform"), (3, 5, 2, 0.4, "uniform"), (200, 150, 3, 0.1, "loose"), (130, 257, 4, 0.05, "uniform"),
          (257, 130, 5, 0.1, "loose"), (90, 300, 7, 0.2, "zipf"), (65, 64, 8, 0.3, "uniform"), (300, 200, 17, 0.05, "loose"), (128, 1000, 33, 0.03, "zipf"), (33, 400, 64, 0.1, "loose"),
          (500, 300, 65, 0.02, "uniform"), (100, 90, 129, 0.2, "zipf"), (64, 64, 257, 0.3, "loose"), (411, 1500, 300, 0.02, "zipf"), (40, 30, 1031, 0.2, "uniform")]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,k,N,density,kind", SHAPES)
def test_forward(m, k, N, density, kind, dtype):
    i = SHAPES.index((m, k, N, density, kind)) + list(TYPES).index(dtype)
    act = list(binding.ACTIVATIONS)[i % 5]
    forward_case(m, k, N, density, kind, TYPES[dtype], act, bias=i % 3 != 1, residual=i % 2 == 0, keep=i % 4 < 2)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N,extra,shift", [(1, 3, 1), (6, 2, 2), (64, 8, 8), (64, 1, 0), (61, 3, 1), (200, 56, 4), (130, 30, 2), (130, 5, 3)])
def test_forward_strides(N, extra, shift, dtype):
    forward_case(150, 170, N, 0.1, "loose", TYPES[dtype], "gelu", True, True, True, extra, shift)


@pytest.mark.parametrize("act", list(binding.ACTIVATIONS))
@pytest.mark.parametrize("dtype", list(TYPES))
def test_activations(act, dtype):
    forward_case(120, 80, 40, 0.3, "uniform", TYPES[dtype], act, True, False, True)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("m,k,N,extra,shift,density", [(1500, 1600, 515, 0, 0, 0.05), (1500, 1600, 515, 5, 0, 0.05), (1500, 1600, 514, 0, 1, 0.02), (3000, 3000, 301, 0, 0, 0.02), (900, 1000, 17, 1, 0, 0.02), (700, 20000, 303, 0, 0, 0.01)])
def test_rows_at_odd_places(m, k, N, extra, shift, density, dtype):
    """An odd number of columns, odd leading dimensions and odd beginnings, where it pays to copy B first and where it does not."""
    forward_case(m, k, N, density, "uniform", TYPES[dtype], "relu", True, True, True, extra, shift)
    values_case(m, k, N, density, "uniform", TYPES[dtype], extra, shift)


def every(list_):
    return [(*shape[:5], dtype) for shape, _ in list_ for dtype in shape[5].split()]


@pytest.mark.parametrize("m,k,N,density,kind,dtype", every(ref.KERNELS))
def test_forward_by_every_kernel(m, k, N, density, kind, dtype):
    """Against products of dense matrices in 64 bits."""
    T = TYPES[dtype]
    print(f"forward: {m} x {k} x {N} {density} {kind} {dtype}", flush=True)
    arrays = csr(m, k, density, m + N, kind)
    A = matrix(m, k, arrays)
    rows = torch.from_numpy(np.repeat(np.arange(m), np.diff(arrays[0]))).to(DEV)
    W = torch.zeros((m, k), dtype=torch.float64, device=DEV)
    W.index_put_((rows, torch.from_numpy(arrays[1]).to(DEV).long()), torch.from_numpy(arrays[2]).to(DEV).double(), accumulate=True)
    M = torch.zeros_like(W)
    M.index_put_((rows, torch.from_numpy(arrays[1]).to(DEV).long()), torch.from_numpy(arrays[2]).to(DEV).double().abs(), accumulate=True)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(m + k)
    B, R = torch.randn((k, N), generator=gen, device=DEV).to(T), torch.randn((m, N), generator=gen, device=DEV).to(T)
    b = torch.randn(m, generator=gen, device=DEV)
    C, Z = torch.full((m, N + 1), 7.0, dtype=T, device=DEV), torch.full((m, N + 3), 7.0, dtype=T, device=DEV)
    binding.gcoo_spdm_epilogue(A, B, bias=b, activation="relu", residual=R, C_out=C[:, :N], Z_out=Z[:, :N])
    z = W @ B.double() + b.double()[:, None]
    off = (torch.from_numpy(np.diff(arrays[0])).to(DEV).double()[:, None] + 2) * ref.F32 * (M @ B.double().abs()) + ref.F32 * z.abs()
    u, least = ref.U[T], ref.LEAST[T]
    ref.check_on_gpu(Z[:, :N], z, off + u * (z.abs() + off) + least, "Z")
    y = z.clamp(min=0) + R.double()
    off = off + ref.F32 * y.abs()
    ref.check_on_gpu(C[:, :N], y, off + u * (y.abs() + off) + least, "C")
    assert torch.all(C[:, N:] == 7.0) and torch.all(Z[:, N:] == 7.0)
    again = binding.gcoo_spdm_epilogue(A, B, bias=b, activation="relu", residual=R)
    assert torch.equal(again, C[:, :N])


@pytest.mark.parametrize("m,k,N,density,kind,dtype", every(ref.VALUES_KERNELS))
def test_grad_values_by_every_kernel(m, k, N, density, kind, dtype):
    T = TYPES[dtype]
    print(f"values: {m} x {k} x {N} {density} {kind} {dtype}", flush=True)
    arrays = csr(m, k, density, m + N, kind)
    A = matrix(m, k, arrays)
    rows, cols = torch.from_numpy(np.repeat(np.arange(m), np.diff(arrays[0]))).to(DEV), torch.from_numpy(arrays[1]).to(DEV).long()
    gen = torch.Generator(device=DEV)
    gen.manual_seed(m + k)
    dZ, B = torch.randn((m, N), generator=gen, device=DEV).to(T), torch.randn((k, N), generator=gen, device=DEV).to(T)
    got = binding.gcoo_spdm_grad_values(A, dZ, B)
    want, off = (dZ.double() @ B.double().t().contiguous())[rows, cols], (N + 2) * ref.F32 * (dZ.double().abs() @ B.double().abs().t().contiguous())[rows, cols]
    ref.check_on_gpu(got, want, off, "dvals")
    assert torch.equal(binding.gcoo_spdm_grad_values(A, dZ, B), got)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,k,N,density,kind,p", [(1000, 900, 333, 0.05, "uniform", 32), (2600, 2600, 520, 0.02, "uniform", 128), (6000, 500, 40, 0.02, "uniform", 8), (20000, 300, 12, 0.01, "uniform", 32), (1500, 2000, 100, 0.03, "zipf", 200)])
def test_forward_large(m, k, N, density, kind, p, dtype):
    forward_case(m, k, N, density, kind, TYPES[dtype], "silu", True, True, True, p=p)


def test_forward_of_a_dense_matrix_and_of_none():
    print("forward: from a dense matrix, without entries, without columns", flush=True)
    rng = np.random.default_rng(5)
    W = normal(rng, 300, 250) * (normal(rng, 300, 250) > 1.0)
    B = normal(rng, 250, 70, dtype=torch.bfloat16)
    y = binding.gcoo_spdm_epilogue(binding.gcoo_from_dense(W, 32), B)
    (want, _), (off, _) = ref.forward(ref.f64(W), np.abs(ref.f64(W)), (ref.f64(W) != 0).sum(1), ref.f64(B), None, "none", None, torch.bfloat16)
    ref.check(y, want, off)
    none = np.zeros(41, np.int32), np.zeros(0, np.int32), np.zeros(0, np.float32)
    for k in (7, 0):
        A = matrix(40, k, none)
        b, R = normal(rng, 40), normal(rng, 40, 9)
        Z = torch.empty_like(R)
        C = binding.gcoo_spdm_epilogue(A, torch.full((k, 9), float("nan"), device=DEV), bias=b, activation="relu", residual=R, Z_out=Z)
        assert torch.equal(Z, b[:, None].expand(40, 9)) and torch.equal(C, Z.clamp(min=0) + R)
        assert binding.gcoo_spdm_grad_values(A, R, torch.zeros((k, 9), device=DEV)).shape == (0,)
    A = matrix(40, 7, none)
    assert binding.gcoo_spdm_epilogue(A, torch.empty((7, 0), device=DEV)).shape == (40, 0)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_values_that_are_not_finite(dtype):
    """A row of B that no entry touches does not reach C; what does, reaches the rows that touch it and no other; a residual's NaN stays in its place."""
    print(f"forward: not finite, {dtype}", flush=True)
    m, k = 60, 90
    arrays = csr(m, k, 0.05, 3)
    arrays[1][arrays[1] == 11] = 12
    for N in (1, 5, 40, 200):
        B = normal(np.random.default_rng(N), k, N).to(TYPES[dtype])
        clean = binding.gcoo_spdm_epilogue(matrix(m, k, arrays), B, activation="silu")
        B[11] = float("nan")
        assert torch.equal(binding.gcoo_spdm_epilogue(matrix(m, k, arrays), B, activation="silu"), clean)
        B[12] = float("inf")
        C = binding.gcoo_spdm_epilogue(matrix(m, k, arrays), B, activation="relu")
        touched = np.zeros(m, bool)
        touched[np.repeat(np.arange(m), np.diff(arrays[0]))[arrays[1] == 12]] = True
        assert torch.isfinite(C[torch.from_numpy(~touched).to(DEV)]).all() and touched.any()
        R = torch.zeros((m, N), dtype=TYPES[dtype], device=DEV)
        R[5, 0] = float("nan")
        B[11:13] = 1.0
        assert torch.isnan(binding.gcoo_spdm_epilogue(matrix(m, k, arrays), B, residual=R)).sum() == 1


# ---- the gradient through the epilogue ----

@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,N,extra,shift", [(1, 1, 0, 0), (5, 1, 0, 0), (900, 1, 2, 1), (33, 7, 0, 0), (64, 64, 0, 0), (31, 200, 8, 8), (17, 1023, 1, 1), (2, 5000, 0, 0), (1, 70001, 0, 0), (1300, 40, 3, 2),
                                              (4000, 16, 0, 0), (300, 2048, 0, 0)])
def test_epilogue_grad(m, N, extra, shift, dtype):
    rng = np.random.default_rng(m + N)
    for act in binding.ACTIVATIONS:
        print(f"epilogue_grad: {m} x {N} {dtype} {act} extra={extra} shift={shift}", flush=True)
        dC = Padded(m, N, TYPES[dtype], extra, shift, normal(rng, m, N, dtype=TYPES[dtype]))
        Z = Padded(m, N, TYPES[dtype], extra, shift, 3.0 * normal(rng, m, N, dtype=TYPES[dtype]))
        to = Padded(m, N, TYPES[dtype], extra, shift)
        dZ, db = binding.gcoo_epilogue_grad(dC.t, Z=Z.t, activation=act, dZ_out=to.t)
        (want, want_b), (off, off_b) = ref.epilogue_grad(ref.f64(dC.t), ref.f64(Z.t), act, TYPES[dtype])
        ref.check(dZ, want, off, "dZ")
        ref.check(db, want_b, off_b, "dbias")
        assert dZ is to.t and to.whole() and Z.whole() and dC.whole()
        inside = dC.t.clone()
        _, db2 = binding.gcoo_epilogue_grad(inside, Z=Z.t, activation=act, dZ_out=inside)
        assert torch.equal(inside, dZ) and torch.equal(db, db2)
        over = Z.t.clone()
        _, db3 = binding.gcoo_epilogue_grad(dC.t, Z=over, activation=act, dZ_out=over)
        assert torch.equal(over, dZ) and torch.equal(db, db3)
    same, db = binding.gcoo_epilogue_grad(dC.t)
    assert same is dC.t


def test_epilogue_grad_far_from_zero():
    print("epilogue_grad: far from zero", flush=True)
    z = torch.tensor([-3e38, -1e20, -1e6, -300.0, -100.0, -50.0, -9.0, -5.5, -0.0, 0.0, 1e-30, 4.0, 5.5, 9.0, 50.0, 100.0, 1e6, 1e20, 3e38], device=DEV)[None, :].contiguous()
    d = torch.ones_like(z)
    for act in binding.ACTIVATIONS:
        with np.errstate(over="ignore", invalid="ignore"):
            want = ref.slope(act, np.clip(ref.f64(z), -400.0, 400.0))
        got, _ = binding.gcoo_epilogue_grad(d, Z=z, activation=act)
        ref.check(got, want, np.full(want.shape, 2.0 ** -19 + 2.0 ** -24), act)
        A = matrix(1, 1, (np.array([0, 1], np.int32), np.zeros(1, np.int32), np.ones(1, np.float32)))
        y = binding.gcoo_spdm_epilogue(A, z, activation=act)
        if act == "none" or act == "relu":
            assert torch.equal(y, z if act == "none" else z.clamp(min=0))
        else:
            want = np.where(ref.f64(z) > 30, ref.f64(z), np.where(ref.f64(z) < -200, 0.0, ref.activate(act, np.clip(ref.f64(z), -400.0, 400.0))))
            # (below -30 the value is z exp(z), whose error is that of the exponential, (1.5 |z| + 2) 2^-24 of it: at z = -50 that is 77 2^-24 = 4.8 2^-20, of 1e-20)
            tail = np.where(ref.f64(z) < -30, (1.5 * np.clip(np.abs(ref.f64(z)), 0.0, 400.0) + 2.0) * 2.0 ** -24, 0.0)
            ref.check(y, want, (tail + 2.0 ** -20 + 2.0 ** -24) * np.abs(want) + 2.0 ** -20 * (np.abs(ref.f64(z)) < 30) * np.abs(ref.f64(z)) + 1e-30, act)
    for T in TYPES.values():
        # (a sum that the type has no number for is stored as infinite)
        z = torch.tensor([[-math.inf, math.inf]], device=DEV, dtype=T)
        for act in binding.ACTIVATIONS:
            want = [1.0, 1.0] if act == "none" else [0.0, 1.0]
            got = binding.gcoo_epilogue_grad(torch.ones_like(z), Z=z, activation=act, dZ_out=torch.empty_like(z))[0].double().cpu()[0]
            # (the logistic functions are taken where their exponential is finite: silu at 80, off by 79 exp(-80) < 2^-109; gelu_tanh at 8, where 2u = 49.3 and (2u)' z = 122: off by 123 exp(-49.3) < 2^-64)
            assert (got - torch.tensor(want, dtype=torch.float64)).abs().max() < 2.0 ** -60, (T, act, got)
    nan = torch.full((1, 1), float("nan"), device=DEV)
    for act in ("silu", "gelu", "gelu_tanh"):
        assert torch.isnan(binding.gcoo_epilogue_grad(torch.ones_like(nan), Z=nan, activation=act)[0]).all()
    assert torch.equal(binding.gcoo_epilogue_grad(torch.empty((3, 0), device=DEV), Z=torch.empty((3, 0), device=DEV), activation="silu")[1], torch.zeros(3, device=DEV))


# ---- the gradient of the stored weights ----

VALUES = [(1, 1, 1, 1.0, "uniform"), (1, 900, 1, 0.5, "uniform"), (60, 1, 9, 1.0, "uniform"), (130, 257, 2, 0.05, "loose"), (257, 130, 5, 0.1, "loose"), (90, 300, 8, 0.2, "zipf"), (65, 64, 16, 0.3, "uniform"),
          (300, 200, 17, 0.05, "loose"), (128, 1000, 33, 0.03, "zipf"), (33, 400, 64, 0.1, "loose"), (500, 300, 65, 0.02, "uniform"), (100, 90, 129, 0.2, "zipf"), (64, 64, 257, 0.3, "loose"),
          (300, 260, 300, 0.3, "loose"), (257, 129, 1031, 0.6, "uniform"), (411, 1500, 300, 0.02, "zipf"), (130, 140, 2100, 1.0, "uniform"), (40, 3000, 500, 0.2, "loose"), (1200, 1300, 777, 0.01, "uniform"),
          (1100, 1029, 515, 0.2, "loose")]


def values_case(m, k, N, density, kind, dtype, extra=0, shift=0, p=32):
    print(f"values: {m} x {k} x {N} {density} {kind} {dtype} extra={extra} shift={shift} p={p}", flush=True)
    arrays = csr(m, k, density, m + N, kind)
    A = matrix(m, k, arrays, p)
    rng = np.random.default_rng(N)
    dZ, B = Padded(m, N, dtype, extra, shift, normal(rng, m, N, dtype=dtype)), Padded(k, N, dtype, extra, shift, normal(rng, k, N, dtype=dtype))
    out = Padded(1, len(arrays[1]), torch.float32, 0, 1)
    got = binding.gcoo_spdm_grad_values(A, dZ.t, B.t, out=out.t[0])
    torch.cuda.synchronize()
    want, off = ref.grad_values(arrays[0], arrays[1], ref.f64(dZ.t), ref.f64(B.t))
    ref.check(got, want, off, "dvals")
    assert out.whole() and dZ.whole() and B.whole()
    assert torch.equal(binding.gcoo_spdm_grad_values(A, dZ.t, B.t), got)
    return A, arrays, dZ.t, B.t, got


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,k,N,density,kind", VALUES)
def test_grad_values(m, k, N, density, kind, dtype):
    values_case(m, k, N, density, kind, TYPES[dtype], p=8 if m % 2 else 100)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N,extra,shift,density", [(1, 3, 1, 0.1), (64, 8, 8, 0.05), (64, 8, 8, 0.5), (61, 3, 1, 0.05), (61, 3, 1, 0.5), (200, 56, 4, 0.5), (130, 5, 3, 0.5), (130, 5, 3, 0.02), (2000, 1, 0, 0.5)])
def test_grad_values_strides(N, extra, shift, density, dtype):
    values_case(200, 210, N, density, "loose", TYPES[dtype], extra, shift)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_grad_values_of_rows_that_are_not_finite(dtype):
    """NaN in a row of B or dZ reaches the entries of that column or row, and no other."""
    for N, density in ((3, 0.1), (70, 0.05), (300, 0.6)):
        A, arrays, dZ, B, got = values_case(150, 160, N, density, "uniform", TYPES[dtype])
        rows = np.repeat(np.arange(150), np.diff(arrays[0]))
        B[13, N - 1] = float("nan")
        dZ[149, 0] = float("nan")
        hit = torch.from_numpy((arrays[1] == 13) | (rows == 149)).to(DEV)
        again = binding.gcoo_spdm_grad_values(A, dZ, B)
        assert torch.isnan(again[hit]).all() and torch.equal(again[~hit], got[~hit])


def test_grad_values_of_a_dense_matrix():
    print("values: from a dense matrix", flush=True)
    rng = np.random.default_rng(8)
    W = normal(rng, 200, 170) * (normal(rng, 200, 170) > 0.5)
    dZ, B = normal(rng, 200, 90), normal(rng, 170, 90)
    cells = ref.f64(W).nonzero()
    want = (ref.f64(dZ)[cells[0]] * ref.f64(B)[cells[1]]).sum(1)
    off = 92 * 2.0 ** -24 * (np.abs(ref.f64(dZ))[cells[0]] * np.abs(ref.f64(B))[cells[1]]).sum(1)
    ref.check(binding.gcoo_spdm_grad_values(binding.gcoo_from_dense(W, 32), dZ, B), want, off)
    assert torch.equal(binding.gcoo_spdm_grad_values(binding.gcoo_from_dense(W, 32), dZ[:, :0], B[:, :0]), torch.zeros(len(want), device=DEV))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_far_apart(dtype):
    """Offsets into B (and dZ) beyond 32 bits."""
    T = TYPES[dtype]
    pitch = 2 ** 30 - 8
    for N in (1, 70, 300):
        print(f"far apart: {dtype} N={N}", flush=True)
        m, k = 9, 11
        arrays = csr(m, k, 0.5, 3)
        A = matrix(m, k, arrays)
        far = torch.empty((k - 1) * pitch + N + 1, dtype=T, device=DEV)
        rng = np.random.default_rng(N)
        near, dZ = normal(rng, k, N, dtype=T), normal(rng, m, N, dtype=T)
        for shift in (0, 1):
            B = far[shift:].as_strided((k, N), (pitch, 1))
            B.copy_(near)
            assert torch.equal(binding.gcoo_spdm_grad_values(A, dZ, B), binding.gcoo_spdm_grad_values(A, dZ, near))
            assert torch.equal(binding.gcoo_spdm_epilogue(A, B, activation="silu"), binding.gcoo_spdm_epilogue(A, near, activation="silu"))
        Z = far.as_strided((m, N), (pitch, 1))
        Z.copy_(dZ)
        assert torch.equal(binding.gcoo_spdm_grad_values(A, Z, near), binding.gcoo_spdm_grad_values(A, dZ, near))


# ---- clipping ----

def clip_reference(tensors, max_norm):
    norm = np.sqrt(sum(float((ref.f64(t) ** 2).sum()) for t in tensors))
    return norm, min(1.0, max_norm / (norm + 1e-6))


@pytest.mark.parametrize("sizes,types", [([1], ["f32"]), ([5, 0, 70000, 3], ["f32", "f32", "bf16", "f16"]), ([65536, 65537, 1, 131073], ["f32", "f16", "bf16", "f32"]), (list(range(1, 201)), ["f32", "bf16"]),
                                         ([300000], ["bf16"]), ([300001], ["f16"])])
@pytest.mark.parametrize("max_norm", [1.0, 1e9, 0.0, float("inf")])
def test_clip(sizes, types, max_norm):
    print(f"clip: {len(sizes)} tensors, {max_norm}", flush=True)
    rng = np.random.default_rng(len(sizes))
    held = [Padded(1, n, TYPES[types[i % len(types)]], 0, i % 9, normal(rng, 1, n)) for i, n in enumerate(sizes)]
    tensors = [h.t[0] for h in held]
    before = [t.clone() for t in tensors]
    norm, factor = clip_reference(tensors, max_norm)
    to = [torch.full_like(t, 3.0) for t in tensors]
    got = binding.gcoo_clip_grad_norm(tensors, max_norm, out=to)
    assert abs(float(got) - norm) <= 2.0 ** -23 * norm
    for t, b, o in zip(tensors, before, to):
        assert torch.equal(t, b)
        want = ref.f64(b) * factor
        u = ref.U[t.dtype]
        ref.check(o, want, ((1 + u) * 2.0 ** -22 + (u if factor < 1.0 else 0.0)) * np.abs(want) + (ref.LEAST[t.dtype] if factor < 1.0 else 0.0))
    in_place = binding.gcoo_clip_grad_norm(tensors, max_norm)
    assert torch.equal(in_place, got) and all(torch.equal(t, o) for t, o in zip(tensors, to)) and all(h.whole() for h in held)


def test_clip_of_large_and_of_not_finite_elements():
    print("clip: large, small and not finite", flush=True)
    for value in (1e30, 1e-30):
        x = torch.full((1000,), value, device=DEV)
        n = binding.gcoo_clip_grad_norm([x], value)
        want = value * np.sqrt(1000.0)
        assert abs(float(n) - want) <= 2.0 ** -22 * want
        factor = min(1.0, value / (want + 1e-6))
        assert torch.allclose(x, torch.full_like(x, value * factor), rtol=1e-6, atol=0.0)
    x, y = torch.ones(10, device=DEV), torch.ones(70000, device=DEV)
    x[3] = float("nan")
    assert torch.isnan(binding.gcoo_clip_grad_norm([x, y], 1.0)) and torch.isnan(x).all() and torch.isnan(y).all()
    x, y = torch.ones(10, device=DEV), torch.ones(70000, device=DEV)
    x[3] = float("inf")
    assert torch.isinf(binding.gcoo_clip_grad_norm([x, y], 1.0)) and torch.isnan(x).sum() == 1 and (y == 0).all()


# ---- together ----

def training_step(m, k, arrays, perm, X, dY, bias, R, act, dtype):
    """One step of a layer: forward, all gradients, clipping.  `arrays`: CSR of the weights on the device; `perm`: where the entries of the transpose are among them, with its row_ptr and columns."""
    A = binding.gcoo_from_csr(m, k, *arrays, 32, known_nnz=True)
    At = binding.gcoo_from_csr(k, m, perm[1], perm[2], arrays[2][perm[0]], 32, known_nnz=True)
    Z = torch.empty((m, X.shape[1]), dtype=dtype, device=DEV)
    Y = binding.gcoo_spdm_epilogue(A, X, bias=bias, activation=act, residual=R, Z_out=Z)
    dZ, db = binding.gcoo_epilogue_grad(dY, Z=Z, activation=act)
    dv = binding.gcoo_spdm_grad_values(A, dZ, X)
    dX = binding.gcoo_spdm_epilogue(At, dZ)
    norm = binding.gcoo_clip_grad_norm([dv, db], 0.5)
    return Y, Z, dZ, dX, dv, db, norm


def transpose(m, k, arrays):
    rows = np.repeat(np.arange(m), np.diff(arrays[0]))
    order = np.lexsort((rows, arrays[1]))
    row_ptr = np.concatenate([[0], np.cumsum(np.bincount(arrays[1], minlength=k))]).astype(np.int32)
    return [torch.from_numpy(x).to(DEV) for x in (order, row_ptr, rows[order].astype(np.int32))]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,k,N,density", [(150, 200, 1, 0.1), (260, 190, 130, 0.1), (300, 310, 64, 0.4)])
def test_a_training_step(m, k, N, density, dtype):
    """Every result against 64 bits, each from what the kernels in front of it gave."""
    print(f"step: {m} x {k} x {N} {density} {dtype}", flush=True)
    T = TYPES[dtype]
    arrays = csr(m, k, density, 77)
    perm = transpose(m, k, arrays)
    rng = np.random.default_rng(1)
    X, dY, R, bias = normal(rng, k, N, dtype=T), normal(rng, m, N, dtype=T), normal(rng, m, N, dtype=T), normal(rng, m)
    Y, Z, dZ, dX, dv, db, norm = training_step(m, k, [torch.from_numpy(x).to(DEV) for x in arrays], perm, X, dY, bias, R, "gelu", T)
    W, M = ref.dense(m, k, *arrays)
    lens = np.diff(arrays[0])
    (y, z), (off_y, off_z) = ref.forward(W, M, lens, ref.f64(X), ref.f64(bias), "gelu", ref.f64(R), T)
    ref.check(Y, y, off_y)
    ref.check(Z, z, off_z)
    (g, gb), (off_g, off_b) = ref.epilogue_grad(ref.f64(dY), ref.f64(Z), "gelu", T)
    ref.check(dZ, g, off_g)
    (dx, _), (off_x, _) = ref.forward(W.T, M.T, np.diff(perm[1].cpu().numpy()), ref.f64(dZ), None, "none", None, T)
    ref.check(dX, dx, off_x)
    v, off_v = ref.grad_values(arrays[0], arrays[1], ref.f64(dZ), ref.f64(X))
    want = np.sqrt((v ** 2).sum() + (gb ** 2).sum())
    spread = np.sqrt((off_v ** 2).sum() + (off_b ** 2).sum()) + 2.0 ** -22 * want
    assert abs(float(norm) - want) <= spread
    factor = min(1.0, 0.5 / (want + 1e-6))
    rel = spread / want + 2.0 ** -22
    ref.check(dv, v * factor, (off_v + rel * np.abs(v)) * factor * (1 + rel))
    ref.check(db, gb * factor, (off_b + rel * np.abs(gb)) * factor * (1 + rel))


def test_gradients_against_differences():
    """sum(dY * Y) changes with X, the values and the bias as the gradients say (fp32; a central difference is off by h^2 and by the rounding of Y over h)."""
    print("step: differences", flush=True)
    m, k, N = 60, 70, 33
    arrays = csr(m, k, 0.2, 5)
    perm = transpose(m, k, arrays)
    rng = np.random.default_rng(2)
    X, dY, bias = normal(rng, k, N), normal(rng, m, N), normal(rng, m)
    dev = [torch.from_numpy(x).to(DEV) for x in arrays]
    A = binding.gcoo_from_csr(m, k, *dev, 32, known_nnz=True)
    At = binding.gcoo_from_csr(k, m, perm[1], perm[2], dev[2][perm[0]], 32, known_nnz=True)
    Z = torch.empty((m, N), device=DEV)
    binding.gcoo_spdm_epilogue(A, X, bias=bias, activation="gelu_tanh", Z_out=Z)
    dZ, db = binding.gcoo_epilogue_grad(dY, Z=Z, activation="gelu_tanh")
    dv, dX = binding.gcoo_spdm_grad_values(A, dZ, X), binding.gcoo_spdm_epilogue(At, dZ)
    h = 2.0 ** -6
    uX, uv, ub = normal(rng, k, N), normal(rng, len(arrays[1])), normal(rng, m)

    def loss(t):
        B = binding.gcoo_from_csr(m, k, dev[0], dev[1], dev[2] + t * uv, 32, known_nnz=True)
        return float((dY.double() * binding.gcoo_spdm_epilogue(B, X + t * uX, bias=bias + t * ub, activation="gelu_tanh").double()).sum())

    got = (loss(h) - loss(-h)) / (2 * h)
    finer = (loss(h / 2) - loss(-h / 2)) / h
    want = float((dv.double() * uv.double()).sum() + (dX.double() * uX.double()).sum() + (db.double() * ub.double()).sum())
    # a halved step leaves a quarter of the error of h^2: twice what the two differ covers what is left of it; Y is of order |z| <= 50, rounded to 2^-24 of that, m N terms of it
    assert abs(finer - want) <= 2 * abs(got - finer) + 50 * 2.0 ** -20 * float(dY.abs().sum()) / h


def test_in_a_graph():
    """A training step captured once and replayed on other inputs, eager work and waits between the replays; two graphs with workspaces of their own."""
    print("graph: a training step", flush=True)
    m, k, N = 400, 500, 260
    arrays = csr(m, k, 0.1, 9)
    perm = transpose(m, k, arrays)
    rng = np.random.default_rng(4)
    for dtype in (torch.bfloat16, torch.float32):
        dev = [torch.from_numpy(x).to(DEV) for x in arrays]
        X, dY, R, bias = normal(rng, k, N, dtype=dtype), normal(rng, m, N, dtype=dtype), normal(rng, m, N, dtype=dtype), normal(rng, m)
        training_step(m, k, dev, perm, X, dY, bias, R, "silu", dtype)
        torch.cuda.synchronize()
        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                out = training_step(m, k, dev, perm, X, dY, bias, R, "silu", dtype)
            graphs.append((g, out))
        for turn in range(4):
            for t in (X, dY, R):
                t.copy_(normal(rng, *t.shape, dtype=dtype))
            dev[2].copy_(normal(rng, len(arrays[2])))
            want = training_step(m, k, dev, perm, X, dY, bias, R, "silu", dtype)
            if turn % 2:
                torch.cuda.synchronize()
            for g, _ in graphs:
                g.replay()
            torch.cuda.synchronize()
            for _, out in graphs:
                assert all(torch.equal(a, b) for a, b in zip(out, want)), turn


def test_on_another_stream():
    print("streams: a layer behind a busy stream", flush=True)
    m, k, N = 700, 800, 300
    arrays = csr(m, k, 0.05, 6)
    A = matrix(m, k, arrays)
    rng = np.random.default_rng(4)
    X, dY = normal(rng, k, N, dtype=torch.bfloat16), normal(rng, m, N, dtype=torch.bfloat16)
    Z = torch.empty((m, N), dtype=torch.bfloat16, device=DEV)

    def calls(stream):
        Y = binding.gcoo_spdm_epilogue(A, X, activation="silu", Z_out=Z, stream=stream)
        dZ, db = binding.gcoo_epilogue_grad(dY, Z=Z, activation="silu", stream=stream)
        dv = binding.gcoo_spdm_grad_values(A, dZ, X, stream=stream)
        return Y, dZ, db, dv, binding.gcoo_clip_grad_norm([dv, db], 1.0, stream=stream)

    want = [t.clone() for t in calls(None)]
    big, copy = torch.randn((4096, 4096), device=DEV), torch.empty((4096, 4096), device=DEV)
    st = torch.cuda.Stream(device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        for _ in range(100):
            copy.copy_(big)
    got = calls(st)
    for _ in range(20):
        torch.empty(3000000, dtype=torch.uint8, device=DEV).fill_(0x5a)      # what the calls gave back is not given out while they still use it
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


class _Nothing:
    """In the place of the extension module: serves no call, so that all go by ctypes."""

    def __getattr__(self, name):
        return (lambda h: binding.lib().gcoo_free(h)) if name == "free" else (lambda *args: None)


def test_same_bits_with_and_without_the_module(monkeypatch):
    print("calls: with and without the module", flush=True)
    m, k, N = 300, 310, 70
    arrays = csr(m, k, 0.1, 12)
    perm = transpose(m, k, arrays)
    rng = np.random.default_rng(6)
    results = []
    for _ in range(2):
        for dtype in TYPES.values():
            gen = np.random.default_rng(7)
            X, dY, R, bias = normal(gen, k, N, dtype=dtype), normal(gen, m, N + 3, dtype=dtype)[:, 1:N + 1], normal(gen, m, N, dtype=dtype), normal(gen, m)
            out = training_step(m, k, [torch.from_numpy(x).to(DEV) for x in arrays], perm, X, dY, bias, R, "gelu", dtype)
            plain = binding.gcoo_epilogue_grad(dY)
            assert plain[0] is dY
            results.append([*out, plain[1], binding.gcoo_clip_grad_norm([X.contiguous(), R], 0.1, out=[torch.empty_like(X), torch.empty_like(R)])])
        monkeypatch.setattr(binding, "_calls", _Nothing())
    for a, b in zip(results[:3], results[3:], strict=True):
        assert all(torch.equal(x, y) for x, y in zip(a, b, strict=True))


@pytest.mark.parametrize("module", [True, False])
def test_refuses(module, monkeypatch):
    print("refusals", flush=True)
    binding.lib()
    if not module:
        monkeypatch.setattr(binding, "_calls", _Nothing())
    arrays = csr(30, 40, 0.2, 1)
    A = matrix(30, 40, arrays)
    freed = matrix(30, 40, arrays)
    freed.free()
    X, dZ = torch.zeros((40, 9), device=DEV), torch.zeros((30, 9), device=DEV)
    wide = torch.zeros((30, 18), device=DEV)
    calls = [lambda: binding.gcoo_spdm_epilogue(A, X.cpu()), lambda: binding.gcoo_spdm_epilogue(A, X.double()), lambda: binding.gcoo_spdm_epilogue(A, X[:-1]), lambda: binding.gcoo_spdm_epilogue(A, X.t().contiguous().t()),
             lambda: binding.gcoo_spdm_epilogue(freed, X), lambda: binding.gcoo_spdm_epilogue(A, X, activation="tanh"), lambda: binding.gcoo_spdm_epilogue(A, X, activation=9),
             lambda: binding.gcoo_spdm_epilogue(A, X, bias=torch.zeros(29, device=DEV)), lambda: binding.gcoo_spdm_epilogue(A, X, bias=torch.zeros(30, device=DEV).half()),
             lambda: binding.gcoo_spdm_epilogue(A, X, residual=dZ.half()), lambda: binding.gcoo_spdm_epilogue(A, X, residual=wide[:, ::2]), lambda: binding.gcoo_spdm_epilogue(A, X, Z_out=dZ[:, :8]),
             lambda: binding.gcoo_spdm_epilogue(A, X, C_out=dZ, Z_out=dZ), lambda: binding.gcoo_spdm_epilogue(A, X, C_out=wide[:, :9], residual=wide.view(60, 9)[::1][:30]),
             lambda: binding.gcoo_epilogue_grad(dZ, activation="silu"), lambda: binding.gcoo_epilogue_grad(dZ, Z=dZ[:, :8], activation="silu"), lambda: binding.gcoo_epilogue_grad(dZ.long()),
             lambda: binding.gcoo_epilogue_grad(dZ[:1].expand(30, 9), Z=dZ, activation="silu"), lambda: binding.gcoo_epilogue_grad(dZ, Z=dZ.half(), activation="silu"),
             lambda: binding.gcoo_spdm_grad_values(A, dZ, X.half()), lambda: binding.gcoo_spdm_grad_values(A, dZ[:-1], X), lambda: binding.gcoo_spdm_grad_values(A, dZ, X[:, :8]),
             lambda: binding.gcoo_spdm_grad_values(A, dZ, X, out=torch.zeros(3, device=DEV)), lambda: binding.gcoo_spdm_grad_values(freed, dZ, X),
             lambda: binding.gcoo_clip_grad_norm([], 1.0), lambda: binding.gcoo_clip_grad_norm([dZ.cpu()], 1.0), lambda: binding.gcoo_clip_grad_norm([wide[:, ::2]], 1.0), lambda: binding.gcoo_clip_grad_norm([dZ], -1.0),
             lambda: binding.gcoo_clip_grad_norm([dZ], float("nan")), lambda: binding.gcoo_clip_grad_norm([dZ, dZ], 1.0), lambda: binding.gcoo_clip_grad_norm([dZ, dZ[3:5]], 1.0),
             lambda: binding.gcoo_clip_grad_norm([dZ], 1.0, out=[dZ.half()]), lambda: binding.gcoo_clip_grad_norm([dZ[:10], dZ[10:20]], 1.0, out=[dZ[10:20], dZ[20:]])]
    for i, call in enumerate(calls):
        with pytest.raises((AssertionError, binding.GcooError, ValueError)):
            call()
            print("accepted", i, flush=True)


# Long rows (of more than 512 entries and eight times the mean), which whole workgroups share: one of them the first row, one the last.
LONG = [(1000, 2000, 0.004), (9000, 2500, 0.002), (17000, 6000, 0.0005)]


def long_rows(m, k, density):
    rng = np.random.default_rng(m)
    mask = rng.random((m, k), dtype=np.float32) < density
    mask[[0, 17, 18, 500, m - 1]] = rng.random((5, k), dtype=np.float32) < 0.95
    cells = np.flatnonzero(mask)
    return workloads.csr_from_cells(m, k, cells, rng.standard_normal(len(cells)).astype(np.float32))


@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,k,density", LONG)
def test_long_rows(m, k, density, dtype, dense):
    print(f"long rows: {m} x {k} {density} {dtype} dense={dense}", flush=True)
    T = TYPES[dtype]
    arrays = long_rows(m, k, density)
    row_ptr, cols, vals = arrays
    lens = np.diff(row_ptr)
    assert lens[m - 1] > max(512, 8 * (len(vals) // m))
    W, M = ref.dense(m, k, *arrays)
    A = binding.gcoo_from_dense(torch.from_numpy(W.astype(np.float32)).to(DEV), 32) if dense else matrix(m, k, arrays)
    rng = np.random.default_rng(k)
    for N in (1, 2, 4, 7, 8, 20, 70, 300):
        B, dZ, R, bias = normal(rng, k, N, dtype=T), normal(rng, m, N, dtype=T), normal(rng, m, N, dtype=T), normal(rng, m)
        C, Z = Padded(m, N, T, 3, 1), Padded(m, N, T, 1, 0)
        binding.gcoo_spdm_epilogue(A, B, bias=bias, activation="silu", residual=R, C_out=C.t, Z_out=Z.t)
        got = binding.gcoo_spdm_grad_values(A, dZ, B)
        torch.cuda.synchronize()
        (want, z), (off, off_z) = ref.forward(W, M, lens, ref.f64(B), ref.f64(bias), "silu", ref.f64(R), T)
        ref.check(C.t, want, off, f"C {N}")
        ref.check(Z.t, z, off_z, f"Z {N}")
        ref.check(got, *ref.grad_values(row_ptr, cols, ref.f64(dZ), ref.f64(B)), f"dvals {N}")
        assert C.whole() and Z.whole()
        assert torch.equal(binding.gcoo_spdm_grad_values(A, dZ, B), got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_long_row_held(dtype):
    """Long rows with few tokens whose B is kept in LDS."""
    m, k = 6000, 4000
    rng = np.random.default_rng(5)
    mask = rng.random((m, k), dtype=np.float32) < 0.1
    mask[[3, 4000]] = True
    mask[[5, 6, m - 1]] = False
    cells = np.flatnonzero(mask)
    arrays = workloads.csr_from_cells(m, k, cells, rng.standard_normal(len(cells)).astype(np.float32))
    assert k > 8 * (len(cells) // m) and len(cells) > 2000000
    A, (W, M), T = matrix(m, k, arrays), ref.dense(m, k, *arrays), TYPES[dtype]
    for N in (1, 3):
        B = normal(rng, k, N, dtype=T)
        C = binding.gcoo_spdm_epilogue(A, B, activation="gelu")
        (want, _), (off, _) = ref.forward(W, M, np.diff(arrays[0]), ref.f64(B), None, "gelu", None, T)
        ref.check(C, want, off, f"C {N}")


# B held in LDS: few tokens and many entries
HELD = [(500, 4000, 1, 0.12, 0, 0), (500, 4000, 1, 0.12, 6, 1), (700, 3000, 2, 0.12, 0, 1), (700, 3000, 2, 0.12, 3, 0), (700, 3000, 3, 0.12, 0, 0), (700, 3000, 4, 0.2, 1, 1), (700, 3000, 5, 0.25, 0, 0), (700, 3000, 7, 0.25, 9, 3),
        (700, 3000, 8, 0.25, 0, 0), (700, 3000, 8, 0.25, 1, 1), (700, 3001, 11, 0.4, 0, 1), (700, 3001, 16, 0.5, 0, 0), (900, 2999, 27, 0.4, 5, 1), (900, 2999, 32, 0.4, 0, 0), (20000, 400, 3, 0.05, 0, 0),
        (300, 9980, 8, 0.1, 0, 0), (200, 19900, 4, 0.1, 0, 1), (130, 39000, 2, 0.1, 0, 0), (65, 79000, 1, 0.1, 0, 1)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,k,N,density,extra,shift", HELD)
def test_forward_held(m, k, N, density, extra, shift, dtype):
    forward_case(m, k, N, density, "uniform" if N % 2 else "loose", TYPES[dtype], "gelu_tanh", True, N % 3 != 0, N % 2 == 0, extra, shift)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_forward_held_of_rows_that_are_not_finite(dtype):
    """NaN and infinities in rows of B that no entry touches, the first and the last among them, and behind its columns, reach nothing; C may be the residual."""
    T, m, k = TYPES[dtype], 400, 3000
    rng = np.random.default_rng(4)
    mask = rng.random((m, k), dtype=np.float32) < 0.5
    mask[:, [0, 77, k - 1]] = False
    mask[5] = False
    cells = np.flatnonzero(mask)
    arrays = workloads.csr_from_cells(m, k, cells, rng.standard_normal(len(cells)).astype(np.float32))
    A, (W, M) = matrix(m, k, arrays), ref.dense(m, k, *arrays)
    for N in (1, 3, 4, 7, 8):
        B = Padded(k, N, T, 2, 1, normal(rng, k, N, dtype=T))
        B.all[B.all == 7.0] = float("nan")
        want, off = ref.forward(W, M, np.diff(arrays[0]), ref.f64(B.t), None, "relu", None, T)
        B.t[0], B.t[77], B.t[k - 1] = float("nan"), float("inf"), -float("inf")
        C = Padded(m, N, T, 1, 1, normal(rng, m, N, dtype=T))
        R = C.t.clone()
        binding.gcoo_spdm_epilogue(A, B.t, activation="relu", residual=C.t, C_out=C.t)
        torch.cuda.synchronize()
        w = want[0] + ref.f64(R)
        ref.check(C.t, w, off[0] + (ref.U[T] + ref.F32) * np.abs(w) + ref.LEAST[T], f"C {N}")
        assert C.whole()
        assert torch.equal(C.t[5], R[5])
