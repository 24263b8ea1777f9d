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


if __name__ == "__main__":
    {f.__name__: f for f in (bounds,)}[sys.argv[1]]()
    print("ok")
