"""Norms and factors at the ends of FP32's range.  The norm that the factor is formed by is the FP32 one: above the range it
is infinite, and the factor zero; a factor below the smallest normal number is a subnormal one, whose bits are fewer."""
import numpy as np
import pytest
import torch

import paper_2606_25759_amd as nf
from tests.test_gpu_norm import factor

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
MAX = float(np.finfo(np.float32).max)


def run(src, dst, max_norm, both):
    plan = nf.norm_plan(src, dst)
    norms, ws = torch.full((1,), -1.0, device=DEV), nf.empty_workspace(nf.nf_grad_norm_workspace_bytes(plan))
    if both:
        nf.nf_grad_norm_clip(plan, max_norm, norms, ws)
    else:
        nf.nf_grad_norm(plan, norms, ws)
        nf.nf_grad_clip(plan, norms, max_norm)
    return float(norms)


@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("blocks", [False, True])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_a_norm_above_the_range_is_infinite(kind, blocks, both):
    n = 3_000_000 if blocks else 4  # sums of many blocks, or of one
    big = torch.finfo(kind).max
    for place in ("f32", "itself"):
        src = torch.full((n,), big, dtype=kind, device=DEV)
        src[1] = -big
        dst = src if place == "itself" else torch.full((n,), 7.0, device=DEV)
        assert np.isposinf(run([src], [dst], 1.0, both))
        assert bool((dst == 0).all())  # and no NaN: there is no infinity among them


@pytest.mark.parametrize("both", [False, True])
def test_just_below_the_range(both):
    """sqrt(n) 2^e, exact: the largest power of two that FP32 has, and a factor that is subnormal."""
    src = torch.full((4,), 2.0 ** 126, device=DEV)
    dst = torch.empty_like(src)
    assert run([src], [dst], 1.0, both) == 2.0 ** 127
    assert torch.equal(dst, torch.full_like(dst, 0.5))  # by 2^-127
    src = torch.tensor([MAX], device=DEV)
    dst = torch.empty_like(src)
    assert run([src], [dst], 3.0, both) == MAX
    by = factor(MAX, 3.0)
    assert 0 < by < np.finfo(np.float32).tiny
    assert float(dst) == float(np.float32(MAX) * by)


@pytest.mark.parametrize("both", [False, True])
def test_a_factor_below_the_smallest_number_is_zero(both):
    src = torch.full((4,), 2.0 ** 120, device=DEV)
    dst = torch.empty_like(src)
    assert run([src], [dst], 2.0 ** -40, both) == 2.0 ** 121
    assert bool((dst == 0).all())  # by 2^-161
