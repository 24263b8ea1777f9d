"""Clipping where the norm, or the factor, is beyond what fp32 holds."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2005_14469_amd import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("n", [2000, 100000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("max_norm", [1.0, 1e-30, 3e38])
def test_a_norm_beyond_fp32(max_norm, dtype, n):
    """Finite elements whose norm fp32 has no number for are scaled to max_norm as any others; the norm is stored as infinite."""
    print(f"clip: norm beyond fp32, {n} {dtype} {max_norm}", flush=True)
    x = torch.full((n,), 3e37, device=DEV).to(dtype)
    x[::2] = -x[::2]
    x[7] = 1.0
    before = x.double()
    norm = math.sqrt(float((before * before).sum()))
    assert norm > 3.5e38 and torch.isinf(binding.gcoo_clip_grad_norm([x], max_norm))
    # (the factor is rounded twice at the most, a product once or twice, the result to the type: 4 2^-24 and the type's; below 2^-126 fp32 has multiples of 2^-149, bf16 of 2^-133)
    want = before * (max_norm / (norm + 1e-6))
    u, least = (2.0 ** -24, 2.0 ** -149) if dtype is torch.float32 else (2.0 ** -8, 2.0 ** -133)
    assert ((x.double() - want).abs() <= (4 * 2.0 ** -24 + u) * want.abs() + least).all()


def test_not_finite_elements_still_reach_everything():
    for value, nan in ((math.inf, False), (math.nan, True)):
        x, y = torch.ones(70000, device=DEV), torch.ones(10, device=DEV)
        x[5] = value
        n = binding.gcoo_clip_grad_norm([x, y], 1.0)
        assert (torch.isnan(n) and torch.isnan(x).all() and torch.isnan(y).all()) if nan else (torch.isinf(n) and torch.isnan(x).sum() == 1 and (y == 0).all())
    # nothing is clipped to an infinite norm
    x = torch.tensor([math.inf, 2.0], device=DEV)
    assert torch.isinf(binding.gcoo_clip_grad_norm([x], math.inf)) and x.tolist() == [math.inf, 2.0]
