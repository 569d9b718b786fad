"""Clipping where the factor leaves float32's normal numbers: the products do not."""
import pytest
import torch

from operator_util import U
from paper_2412_07752_amd import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value,max_norm", [(3e38, 1.0), (3e38, 1e-6), (3e38, 1e-20), (1e30, 1e-10), (2e20, 1e-22)])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("count", [5, 10_000, 20_000_000])
def test_factors_below_the_smallest_normal_number(value, max_norm, in_place, count):
    """out = max_norm / norm * g to a few roundings (two of the factor, one of the product), wherever out itself is a normal number."""
    grads = [torch.full((count,), value, device="cuda"), torch.full((33,), -value, device="cuda", dtype=torch.bfloat16), torch.full((3,), 1e-3, device="cuda")]
    total = sum(g.numel() * g[0].double().item() ** 2 for g in grads)
    factor = max_norm / total ** 0.5
    out = grads if in_place else [torch.full_like(g, 7.0) for g in grads]
    want = [g[0].double().item() * factor for g in grads]
    norm = api.flashrnn_grad_clip(grads, max_norm, out=None if in_place else out)
    assert norm.item() == float("inf") if total ** 0.5 > torch.finfo(torch.float32).max * (1 + U) else abs(norm.item() - total ** 0.5) <= 2 * U * total ** 0.5
    for o, w in zip(out, want):
        unit = U if o.dtype == torch.float32 else 2.0 ** -8
        for got in (o.min().item(), o.max().item()):
            assert abs(got - w) <= (4 * U + unit) * abs(w) + 2.0 ** -126 * (abs(w) < 2.0 ** -126), (got, w)
