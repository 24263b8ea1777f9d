"""The gradient of the stored weights over so many columns that its sums are joined in several groups."""
import pytest

torch = pytest.importorskip("torch")

from paper_2005_14469_amd import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("m,k,N,entries,tile", [(12000, 12000, 3101, 5800000, 256), (8000, 8000, 22000, 3200000, 512), (3000, 3000, 100002, 700000, 1024), (9000, 12000, 12003, 4100000, 256)])
def test_groups_of_tiles(m, k, N, entries, tile):
    """Against dense products in 64 bits; columns in no order, some twice, the first rows ten times as long as the others."""
    print(f"values: {m} x {k} x {N}, {entries} entries", flush=True)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(N)
    rows = torch.randint(m, (entries,), generator=gen, device=DEV)
    rows[:entries // 50] %= 100
    rows = rows.sort().values
    cols = torch.randint(k, (entries,), generator=gen, device=DEV)
    row_ptr = torch.zeros(m + 1, dtype=torch.int32, device=DEV)
    row_ptr[1:] = torch.bincount(rows, minlength=m).cumsum(0)
    A = binding.gcoo_from_csr(m, k, row_ptr, cols.int(), torch.ones(entries, device=DEV), 32, known_nnz=True)
    dZ, B = torch.randn((m, N), generator=gen, device=DEV), torch.randn((k, N), generator=gen, device=DEV)
    # (tiles of so many bytes of a row of B: less work than a sum for each, a copy of B aside, is more than one group)
    assert binding.lib().gcoo_spdm_grad_values_bytes(A.handle, dZ.data_ptr(), N, B.data_ptr(), N, N, binding.GCOO_F32) - 4 * k * (N + 63) < 4 * entries * (4 * N // tile)
    got = binding.gcoo_spdm_grad_values(A, dZ, B)
    assert torch.equal(binding.gcoo_spdm_grad_values(A, dZ, B), got)
    want, size = torch.zeros((m, k), dtype=torch.float64, device=DEV), torch.zeros((m, k), dtype=torch.float64, device=DEV)
    for j in range(0, N, 8192):
        z, b = dZ[:, j:j + 8192].double(), B[:, j:j + 8192].double()
        want += z @ b.t().contiguous()
        size += z.abs() @ b.abs().t().contiguous()
    assert ((got.double() - want[rows, cols]).abs() <= (N + 2) * 2.0 ** -24 * size[rows, cols]).all()
