"""The host code of the operators of a sparse layer run without a GPU, on the HIP calls of tests/host/hip_on_host.cpp (see host_calls.py): what is refused, before anything is
launched.  `python -m tests.layer_calls NAME`."""
import ctypes as C
import sys

from tests.host_calls import EHIP, EINVAL, ENOMEM, OK, Host

F32, BF16, F16 = 0, 1, 2
AT = 1 << 40                    # addresses that nothing reads
i64, i32, vp, sz, ci = C.c_int64, C.c_int32, C.c_void_p, C.c_size_t, C.c_int


class Epilogue(C.Structure):
    _fields_ = [("type", i32), ("activation", i32), ("bias", vp), ("residual", vp), ("ldr", i64), ("Z", vp), ("ldz", i64)]


class Gradient(C.Structure):
    _fields_ = [("data", vp), ("out", vp), ("count", i64), ("type", i32)]


class Layer(Host):
    def __init__(self):
        super().__init__()
        for name, res, args in [("gcoo_spdm_epilogue_bytes", sz, [vp, vp, i64, i64, vp, vp, i64]), ("gcoo_spdm_epilogue", ci, [vp, vp, i64, i64, vp, vp, i64, vp, sz, vp]),
                                ("gcoo_epilogue_grad_bytes", sz, [i64, i64]), ("gcoo_epilogue_grad", ci, [i64, i64, ci, ci, vp, i64, vp, i64, vp, i64, vp, vp, sz, vp]),
                                ("gcoo_spdm_grad_values_bytes", sz, [vp, vp, i64, vp, i64, i64, ci]), ("gcoo_spdm_grad_values", ci, [vp, vp, i64, vp, i64, i64, ci, vp, vp, sz, vp]),
                                ("gcoo_clip_grad_norm_bytes", sz, [vp, i64]), ("gcoo_clip_grad_norm", ci, [vp, i64, C.c_float, vp, vp, sz, vp])]:
            f = getattr(self.L, name)
            f.restype, f.argtypes = res, args

    def refused(self, status, what):
        assert status == EINVAL, (what, status)
        assert not self.launches(), what

    def forward(self, h, N=9, ldb=None, ldc=None, B=AT, Cp=2 * AT, work=4 * AT, bytes=1 << 50, e=None, **kw):
        e = Epilogue(**kw) if e is None else e
        ldb, ldc = N if ldb is None else ldb, N if ldc is None else ldc
        return self.L.gcoo_spdm_epilogue(h, B, ldb, N, C.byref(e), Cp, ldc, work, bytes, None)

    def forward_bytes(self, h, N=9, ldb=None, ldc=None, B=AT, Cp=2 * AT, **kw):
        return self.L.gcoo_spdm_epilogue_bytes(h, B, N if ldb is None else ldb, N, C.byref(Epilogue(**kw)), Cp, N if ldc is None else ldc)

    def grad(self, m=30, N=9, type=F32, act=1, Z=AT, ldz=9, dC=2 * AT, lddc=9, dZ=3 * AT, lddz=9, db=5 * AT, work=4 * AT, bytes=1 << 50):
        return self.L.gcoo_epilogue_grad(m, N, type, act, Z, ldz, dC, lddc, dZ, lddz, db, work, bytes, None)

    def values(self, h, dZ=AT, lddz=9, B=2 * AT, ldb=9, N=9, type=F32, out=3 * AT, work=4 * AT, bytes=1 << 50):
        return self.L.gcoo_spdm_grad_values(h, dZ, lddz, B, ldb, N, type, out, work, bytes, None)

    def clip(self, *tensors, max_norm=1.0, norm=AT - 4, work=4 * AT, bytes=1 << 50):
        arr = (Gradient * max(1, len(tensors)))(*[Gradient(*t) for t in tensors])
        return self.L.gcoo_clip_grad_norm(arr, len(tensors), max_norm, norm, work, bytes, None)


def refusals():
    H = Layer()
    h = H.matrix(30, 40, 200, 32)
    none = H.matrix(30, 40, 0, 32)
    H.log()
    assert H.forward(h) == OK and H.launches()
    H.refused(H.L.gcoo_spdm_epilogue(None, AT, 9, 9, C.byref(Epilogue()), 2 * AT, 9, 4 * AT, 1 << 50, None), "no matrix")
    H.refused(H.L.gcoo_spdm_epilogue(h, AT, 9, 9, None, 2 * AT, 9, 4 * AT, 1 << 50, None), "no epilogue")
    for kw in (dict(type=3), dict(type=-1), dict(activation=5), dict(activation=-1), dict(ldb=8), dict(ldc=8), dict(ldb=1 << 30), dict(N=-1), dict(N=1 << 31, ldb=1 << 31, ldc=1 << 31), dict(B=None), dict(Cp=None),
               dict(residual=3 * AT, ldr=8), dict(Z=3 * AT, ldz=8), dict(residual=2 * AT, ldr=10), dict(Z=2 * AT, ldz=9), dict(bias=AT + 2), dict(B=AT + 2), dict(B=AT + 1, type=BF16), dict(Cp=AT + 3, type=F16),
               dict(residual=AT + 1, ldr=9, type=F16), dict(Z=AT + 2, ldz=9),
               dict(B=2 * AT), dict(Z=AT, ldz=9), dict(residual=3 * AT, ldr=9, Z=3 * AT, ldz=9)):
        H.refused(H.forward(h, **kw), kw)
    need = H.forward_bytes(h, type=BF16)
    if need:
        assert H.forward(h, type=BF16, bytes=need) == OK and H.launches()
        assert H.forward(h, type=BF16, bytes=need - 1) == ENOMEM and not H.launches()
        H.refused(H.forward(h, type=BF16, work=None), "no work")
        H.refused(H.forward(h, type=BF16, work=4 * AT + 128), "work at an odd place")
    assert H.forward(h, N=0) == OK and not H.launches()
    assert H.forward(none, B=None, work=None, bytes=0) == OK and len(H.launches()) == 1
    assert H.forward(h, residual=2 * AT, ldr=9) == OK and H.launches()

    assert H.grad() == OK and H.launches()
    for kw in (dict(m=-1), dict(N=-1), dict(m=1 << 31), dict(N=1 << 31, ldz=1 << 31, lddc=1 << 31, lddz=1 << 31), dict(type=3), dict(act=5), dict(act=-1), dict(lddc=8), dict(ldz=8), dict(lddz=8), dict(dC=None), dict(Z=None),
               dict(dC=AT + 2), dict(Z=AT + 1, type=BF16), dict(dZ=AT + 1, type=F16), dict(db=AT + 2), dict(dZ=2 * AT, lddz=10), dict(dZ=AT, lddz=10)):
        H.refused(H.grad(**kw), kw)
    assert H.grad(dZ=AT) == OK and H.launches()
    # (more threads than a launch takes; a wide matrix of as many rows has lanes of its own for every row)
    assert H.grad(m=1 << 28, N=1) == EHIP and not H.launches()
    assert H.grad(m=(1 << 28) - 16, N=1) == OK and H.launches()
    assert H.grad(m=1 << 24, N=5000, ldz=5000, lddc=5000, lddz=5000) == EHIP and not H.launches()
    assert H.grad(act=0, Z=None, ldz=0, dZ=None, lddz=0) == OK and H.launches()
    wide = dict(m=1, N=70001, ldz=70001, lddc=70001, lddz=70001)
    need = H.L.gcoo_epilogue_grad_bytes(1, 70001)
    assert need > 0 and H.grad(**wide, bytes=need) == OK and len(H.launches()) == 2
    assert H.grad(**wide, bytes=need - 1) == ENOMEM and not H.launches()
    for kw in (dict(m=0), dict(dZ=None, db=None), dict(N=0, dC=None, Z=None, db=None)):
        assert H.grad(**kw) == OK and not H.launches(), kw
    assert H.grad(N=0, dC=None, Z=None) == OK and len(H.launches()) == 1

    assert H.values(h) == OK and H.launches()
    H.refused(H.values(None), "no matrix")
    for kw in (dict(type=3), dict(N=-1), dict(lddz=8), dict(ldb=8), dict(lddz=1 << 30), dict(ldb=1 << 30), dict(dZ=None), dict(B=None), dict(out=None), dict(dZ=AT + 2), dict(B=AT + 1, type=F16), dict(out=AT + 2)):
        H.refused(H.values(h, **kw), kw)
    assert H.values(none, dZ=None, B=None, out=None) == OK and not H.launches()

    t = (AT, AT, 100, F32)
    assert H.clip(t) == OK and len(H.launches()) == 1
    for tensors in ([(AT, AT, -1, F32)], [(AT, AT, 10, 3)], [(None, AT, 10, F32)], [(AT, None, 10, F32)], [(AT + 2, AT + 2, 10, F32)], [(AT, AT + 1, 10, F16)], [t, t], [t, (AT + 396, AT + 396, 10, F32)],
                    [(AT, AT + 4, 100, F32)], [(AT, 2 * AT, 100, F32), (2 * AT + 8, 3 * AT, 10, F32)], [(AT, 2 * AT, 100, F32), (3 * AT, 2 * AT + 198, 10, BF16)], [(AT, AT, 1 << 61, F32)], [(AT, AT, 1 << 50, F32)]):
        H.refused(H.clip(*tensors), tensors)
    for kw in (dict(norm=None), dict(norm=AT + 2), dict(norm=AT + 396), dict(max_norm=-1.0), dict(max_norm=float("nan"))):
        H.refused(H.clip(t, **kw), kw)
    assert H.clip((AT, 2 * AT, 100, F32), (AT, 3 * AT, 100, F32), (AT + 400, AT + 400, 5, F32)) == OK and H.launches()      # (read twice, written once each)
    assert H.clip((None, None, 0, F32), max_norm=float("inf"), work=None, bytes=0) == OK and len(H.launches()) == 1
    assert H.clip(bytes=0, work=None) == OK and len(H.launches()) == 1
    H.refused(H.L.gcoo_clip_grad_norm(None, 1, 1.0, AT, AT, 1 << 50, None), "no list")
    many = (AT, AT, 1000000, F32)
    need = H.L.gcoo_clip_grad_norm_bytes((Gradient * 1)(Gradient(*many)), 1)
    assert 0 < need and H.clip(many, norm=AT - 4, bytes=need) == OK and len(H.launches()) == 2
    assert H.clip(many, bytes=need - 1) == ENOMEM and not H.launches()
    H.refused(H.clip(many, work=None), "no work")


def kernels():
    """The shapes of layer_reference.KERNELS launch the kernels that they are there for."""
    from tests import layer_reference as ref
    from paper_2005_14469_amd import workloads
    H = Layer()
    types = {"f32": F32, "bf16": BF16, "f16": F16}
    for shapes, call in ((ref.KERNELS, "forward"), (ref.VALUES_KERNELS, "values")):
        for (m, k, N, density, kind, dtypes), name in shapes:
            nnz = len(workloads.zipf_rows(m, k, 1, m + N, row_max=min(k, 3000)).vals) if kind == "zipf" else int(density * m * k * (2 / 3 if kind == "loose" else 1) + (64 * 0.9 * k if kind == "heavy" else 0))
            h = H.matrix(m, k, nnz, 32)
            for dtype in dtypes.split():
                H.log()
                rc = H.forward(h, N=N, type=types[dtype]) if call == "forward" else H.values(h, N=N, lddz=N, ldb=N, type=types[dtype])
                launched = H.launches()
                assert rc == OK and any(name.format(ref.MANGLED[dtype]) in x for x in launched), ((m, k, N, density, kind, dtype), name, launched)


def a_launch_that_fails():
    H = Layer()
    h = H.matrix(30, 40, 200, 32)
    H.set("hipGetLastError", 1)
    for call in (lambda: H.forward(h), lambda: H.forward(h, type=F16), H.grad, lambda: H.values(h), lambda: H.clip((AT, AT, 100, F32))):
        assert call() == EHIP
    H.set("hipGetLastError", 0)


def launches_of_clipping():
    """Many tensors are as many launches as their descriptions fill; the norm is written once."""
    H = Layer()
    for n, launches in ((1, 1), (6, 1), (7, 2), (80, 2), (81, 4), (400, 10)):
        assert H.clip(*[(AT + 4096 * i, AT + 4096 * i, 1 + i, F32) for i in range(n)]) == OK
        assert len(H.launches()) == launches, n
    assert H.clip(*[(AT + 4096 * i, AT + 4096 * i, i % 2, F32) for i in range(160)]) == OK and len(H.launches()) == 2
    for count, launches in ((6 * 4096, 1), (6 * 4096 + 1, 2)):
        assert H.clip((AT, AT, count, F32)) == OK and len(H.launches()) == launches


if __name__ == "__main__":
    {f.__name__: f for f in (refusals, kernels, a_launch_that_fails, launches_of_clipping)}[sys.argv[1]]()
    print("ok")
