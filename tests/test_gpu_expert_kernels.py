"""Every product kernel with results of 16 bits and of 32, and with more experts than a wavefront has lanes.
test_expert_coverage.py holds what the lists here and in the other tests of them reach."""
import pytest
import torch

import paper_2606_25759_amd as nf
from tests.test_gpu_expert import OTHER_PRODUCTS, TYPES, check_grad, check_product

pytestmark = pytest.mark.gpu

@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("f32", "f16")])
@pytest.mark.parametrize("W,E,T,n,k,extra", OTHER_PRODUCTS)
def test_results_of_16_bits(W, E, T, n, k, extra, kind, out, back):
    check_product(W, E, T, n, k, back, kind, out, extra=extra, seed=n + k)


MANY_EXPERTS = [  # W, E, T, n, k, extra (n and k the other way round where transposed)
    (2, 66, 100, 64, 64, 0), (2, 66, 700, 64, 64, 0), (1, 130, 900, 72, 40, 0), (2, 66, 6000, 64, 64, 0),
    (2, 66, 14_000, 64, 64, 0), (2, 66, 20_000, 264, 40, 0), (2, 66, 100, 63, 61, 1), (1, 200, 700, 61, 66, 1),
    (2, 66, 6000, 65, 63, 1), (2, 66, 20_000, 261, 37, 0), (1, 4096, 300, 8, 16, 0)]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("W,E,T,n,k,extra", MANY_EXPERTS)
def test_more_experts_than_lanes(W, E, T, n, k, extra, kind, out, back):
    check_product(W, E, T, *((k, n) if back else (n, k)), back, kind, out, extra=extra, seed=E + T,
                  offsets=torch.int64 if T % 3 else torch.int32)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kind", list(TYPES))
def test_many_experts_of_edges(kind, back):
    """Experts of no row, of one, of a tile's rows and of one more, where a lane has several."""
    for each in ([0, 1, 31, 32, 33], [127, 0, 0, 128, 129], [0, 0, 0, 255, 257]):
        sizes = [(each * 16)[:79]]
        check_product(1, 79, sum(sizes[0]) + 7, 72, 88, back, kind, "f32", sizes=sizes, start=4)


MANY_SHARED = [(1, 66, 131_072, 64, 64), (1, 100, 131_072, 61, 47)]  # W, E, T, n, k: tokens shared, whatever the type
MANY_WIDE = [(1, 70, 500, 512, 512), (1, 66, 1000, 1024, 1024)]
MANY_GRADS = [(2, 70, 600, 100, 72), (1, 130, 3000, 40, 37)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("W,E,T,n,k", MANY_SHARED)
def test_grad_shared_tokens_of_many_experts(W, E, T, n, k, kind):
    """Sums of several experts a lane to where a share's sums are, and k_join's over more experts than lanes."""
    assert nf.nf_expert_grad_workspace_bytes(W, T, E, n, k) > 0
    check_grad(W, E, T, n, k, kind, lead=1, seed=E)
    sizes = [[0, 3, 9000, 1, 0, 257] * (E // 6) + [0] * (E % 6)]
    assert sum(sizes[0]) <= T + 60_000
    check_grad(W, E, sum(sizes[0]) + 5, n, k, kind, sizes=sizes, start=5, accumulate=True, seed=1)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("W,E,T,n,k", MANY_WIDE)
def test_grad_wide_tiles_of_many_experts(W, E, T, n, k, kind):
    check_grad(W, E, T, n, k, kind, lead=3, seed=E)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("W,E,T,n,k", MANY_GRADS)
def test_grad_of_many_experts(W, E, T, n, k, kind, accumulate):
    check_grad(W, E, T, n, k, kind, accumulate=accumulate, seed=T)
