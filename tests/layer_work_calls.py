"""How much work memory the operators of a sparse layer ask for, and what they do with less, on the host (see layer_calls.py).  `python -m tests.layer_work_calls NAME`."""
import ctypes as C
import sys

from tests.host_calls import ENOMEM, OK
from tests.layer_calls import AT, BF16, F16, F32, Epilogue, Layer

SIZE = {F32: 4, BF16: 2, F16: 2}


def values_bytes(H, h, N, type, ldb=None, lddz=None):
    return H.L.gcoo_spdm_grad_values_bytes(h, AT, N if lddz is None else lddz, 2 * AT, N if ldb is None else ldb, N, type)


def bounds():
    """The sums of the parts that the gradient of the values joins stay below a gigabyte, or 32 bytes per entry, however many columns there are; a copy of B is one, and where the tiles of a row begin is a word for each."""
    H = Layer()
    for m, k, nnz in ((14000, 14000, 16700000), (14000, 14000, 5900000), (8000, 8000, 6400000), (8000, 8000, 320000), (20000, 20000, 800000), (12000, 12000, 5760000), (300, 200000, 3000000), (100000, 1000, 9000000)):
        h = H.matrix(m, k, nnz, 32)
        for type in SIZE:
            for N in (8, 300, 2653, 8000, 65000, 500001):
                most = max(1 << 30, 32 * nnz) + SIZE[type] * k * (N + 63) + 4 * m * ((k + 127) // 128 + 1) + 1024
                got = values_bytes(H, h, N, type)
                assert got <= most, (m, k, nnz, N, type, got, most)


# (m, k, N, entries, type, leading dimension): what asks for work memory, and what is launched with it
FORWARD = [((4000, 4000, 4000, 800000, BF16, 4000), "layer_widen"), ((6000, 6000, 6001, 720000, F16, 6001), "layer_widen"), ((6000, 6000, 500, 1512000, BF16, 500), "layer_realign"),
           ((6000, 6000, 301, 1512000, F32, 301), "layer_realign"), ((3000, 3000, 301, 180000, F16, 301), "layer_realign")]
VALUES = [((4000, 3900, 300, 3120000, BF16, 300), "values_tiles"), ((1100, 1030, 1500, 453000, F32, 1500), "values_join"), ((1000, 12000, 1500, 36000, F32, 1500), "values_join"),
          ((6000, 6000, 500, 1512000, F32, 500), "layer_realign"), ((5000, 4000, 2001, 200000, F16, 2001), "layer_realign"), ((12000, 12000, 8000, 5760000, F32, 8000), "values_join")]


def too_little():
    """As much as was asked for is taken, a byte less, none, or memory at an odd place is refused, and nothing is launched."""
    H = Layer()
    for shapes, product in ((FORWARD, True), (VALUES, False)):
        for (m, k, N, nnz, type, ld), launched in shapes:
            h = H.matrix(m, k, nnz, 32)
            need = H.forward_bytes(h, N=N, ldb=ld, type=type) if product else values_bytes(H, h, N, type)

            def call(work=4 * AT, bytes=need):
                H.log()
                if product:
                    return H.forward(h, N=N, ldb=ld, type=type, work=work, bytes=bytes)
                return H.values(h, N=N, lddz=N, ldb=ld, type=type, work=work, bytes=bytes)

            case = (m, k, N, nnz, type)
            assert need > 0, case
            assert call() == OK and any(launched in x for x in H.launches()), case
            assert call(bytes=need - 1) == ENOMEM and not H.launches(), case
            assert call(bytes=0) == ENOMEM and not H.launches(), case
            H.refused(call(work=None), case)
            H.refused(call(work=4 * AT + 128), case)


def groups():
    """A group of tiles is a launch and one that joins its sums; 12000 columns more are more groups, not more work."""
    H = Layer()
    h = H.matrix(12000, 12000, 5760000, 32)
    needs = []
    for N in (8000, 20000, 32000):
        H.log()
        assert H.values(h, N=N, lddz=N, ldb=N) == OK
        names = ["join" if "values_join" in x else "entries" for x in H.launches() if "values_" in x]
        assert len(names) >= 4 and names == ["entries", "join"] * (len(names) // 2), names
        needs.append(values_bytes(H, h, N, F32))
    assert max(needs) <= 1 << 30, needs


if __name__ == "__main__":
    {f.__name__: f for f in (bounds, too_little, groups)}[sys.argv[1]]()
    print("ok")
