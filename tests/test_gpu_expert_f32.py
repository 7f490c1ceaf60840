"""FP32 products and gradients where they go by rules of their own: results narrow and sums long, tokens shared that 16 bits
would not share.  test_expert_f32_paths.py holds what the lists here reach."""
import pytest

from tests.test_gpu_expert import check_grad, check_product

pytestmark = pytest.mark.gpu

NARROW_RESULTS = [  # W, E, T, n, k, extra (n and k the other way round where transposed)
    (1, 3, 3000, 19, 1300, 0), (1, 2, 2600, 24, 1301, 1), (2, 2, 1500, 80, 1027, 0)]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kind,out", [("f32", "f32"), ("f32", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("W,E,T,n,k,extra", NARROW_RESULTS)
def test_narrow_results(W, E, T, n, k, extra, kind, out, back):
    check_product(W, E, T, *((k, n) if back else (n, k)), back, kind, out, extra=extra, seed=T)


F32_SHARED = [  # W, E, T, n, k: the first three are shared in FP32 only
    (6, 42, 13_462, 116, 23), (1, 10, 2200, 1616, 52), (4, 5, 2673, 596, 16), (1, 32, 32_768, 128, 132), (1, 2, 1300, 600, 632)]


@pytest.mark.parametrize("W,E,T,n,k", F32_SHARED)
def test_grad_shared_tokens_of_f32(W, E, T, n, k):
    check_grad(W, E, T, n, k, "f32", lead=5, gap=3, seed=T)
    check_grad(W, E, T, n, k, "f32", accumulate=True, seed=T)
