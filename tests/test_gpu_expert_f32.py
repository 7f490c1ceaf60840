"""FP32 products and gradients where they go by rules of their own: results narrow and sums long, tokens shared that 16 bits
would not share.  test_expert_f32_paths.py holds what the lists here reach."""
import pytest
import torch

import paper_2606_25759_amd as nf
from tests.test_gpu_expert import DEV, TYPES, check_grad, check_product, close

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


SHIFTED = [(40, 96, 72), (900, 256, 36), (3000, 520, 264), (3000, 133, 131)]  # T, n, k of two experts


def shifted(t, by):
    """The same values `by` elements behind an aligned address, NaN around them."""
    flat = torch.full((t.numel() + 8,), float("nan"), dtype=t.dtype, device=DEV)
    flat[by:by + t.numel()] = t.reshape(-1)
    return flat[by:by + t.numel()].view(t.shape)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("by", [(1, 0, 0), (0, 1, 0), (0, 0, 1), (3, 2, 1)])
@pytest.mark.parametrize("T,n,k", SHIFTED)
def test_places_aligned_to_their_elements_only(T, n, k, by, kind):
    g = torch.Generator().manual_seed(T)
    rand = lambda *s: torch.randn(*s, generator=g).to(TYPES[kind]).to(DEV)  # noqa: E731
    x, dy, w = shifted(rand(T, k), by[0]), shifted(rand(T, n), by[2]), shifted(rand(2, n, k), by[1])
    cut = T // 3
    off = torch.tensor([0, cut, T], dtype=torch.int32, device=DEV)
    y, dx, rows = (torch.empty(*s, device=DEV) for s in ((T, n), (T, k), (1, 2 * n * k + 1)))
    nf.nf_expert_product(x, w, off, y)
    nf.nf_expert_product(dy, w, off, dx, transposed=True)
    nf.nf_expert_grad(dy, x, off, rows, 1, nf.empty_workspace(nf.nf_expert_grad_workspace_bytes(1, T, 2, n, k)))
    for e, at in ((0, slice(0, cut)), (1, slice(cut, T))):
        a, b, m = x[at].double(), dy[at].double(), w[e].double()
        turned, t = m.t().contiguous(), b.t().contiguous()
        close(y[at], a @ turned, a.abs() @ turned.abs(), k)
        close(dx[at], b @ m, b.abs() @ m.abs(), n)
        close(rows[0, 1 + e * n * k:1 + (e + 1) * n * k].view(n, k), t @ a, t.abs() @ a.abs(), at.stop - at.start)
