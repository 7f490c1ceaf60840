"""Rows further apart than 2^20 elements: a tile's offsets would pass what a load straight into LDS can take, so they go by
registers, in every tile (test_expert_f32_paths.py says which these take)."""
import pytest
import torch

import paper_2606_25759_amd as nf
from tests.test_gpu_expert import TYPES, close, offsets_of

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
FAR = (1 << 20) + 4


def far_rows(g, rows, cols, kind):
    """[rows, cols] with its rows FAR apart and NaN between them."""
    big = torch.full((rows * FAR,), float("nan"), dtype=kind, device=DEV)
    t = big.as_strided((rows, cols), (FAR, 1))
    t.copy_(torch.randn(rows, cols, generator=g))
    return t


def near_rows(g, rows, cols, kind):
    return torch.randn(rows, cols, generator=g).to(kind).to(DEV)


# E = 1 matrix with far rows; T, n, k: tiles of 32, of 128 x 32, of 128 (of FP32)
MATRICES = [(20, 40, 36, False), (3000, 130, 20, False), (66_000, 130, 16, False), (20, 36, 40, True), (3000, 20, 131, True),
            (44_000, 20, 260, True)]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("T,n,k,back", MATRICES)
def test_product_of_a_far_matrix(T, n, k, back, kind):
    g = torch.Generator().manual_seed(n)
    w = far_rows(g, n, k, TYPES[kind])
    x = near_rows(g, T, n if back else k, TYPES[kind])
    y = torch.full((T, k if back else n), 7.0, device=DEV)
    nf.nf_expert_product(x, w.unsqueeze(0), torch.tensor([1, T - 2], dtype=torch.int32, device=DEV), y, transposed=back)
    m = w.double() if back else w.double().t().contiguous()
    rows = x[1:T - 2].double()
    close(y[1:T - 2], rows @ m, rows.abs() @ m.abs(), n if back else k)
    assert bool((y[:1] == 7).all()) and bool((y[T - 2:] == 7).all())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("back", [False, True])
def test_product_of_far_tokens(back, kind):
    g = torch.Generator().manual_seed(3)
    T, E, n, k = 150, 3, 40, 33
    x = far_rows(g, T, n if back else k, TYPES[kind])
    w = near_rows(g, E * n, k, TYPES[kind]).view(E, n, k)
    off = offsets_of([[70, 0, 77]])
    y = torch.full((T, k if back else n), 7.0, device=DEV)
    nf.nf_expert_product(x, w, off, y, transposed=back)
    for at, e in ((slice(0, 70), 0), (slice(70, 147), 2)):
        m = w[e].double() if back else w[e].double().t().contiguous()
        rows = x[at].double()
        close(y[at], rows @ m, rows.abs() @ m.abs(), n if back else k)
    assert bool((y[147:] == 7).all())


@pytest.mark.parametrize("which", ["dy", "x"])
@pytest.mark.parametrize("T,n,k", [(60, 100, 72), (500, 70, 96)])  # FP32's tokens of the second are shared
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_grad_of_far_tokens(kind, T, n, k, which):
    g = torch.Generator().manual_seed(T)
    dy = (far_rows if which == "dy" else near_rows)(g, T, n, TYPES[kind])
    x = (far_rows if which == "x" else near_rows)(g, T, k, TYPES[kind])
    off = torch.tensor([2, T - 1], dtype=torch.int64, device=DEV)
    rows = torch.full((1, n * k + 4), 7.0, device=DEV)
    ws = nf.empty_workspace(nf.nf_expert_grad_workspace_bytes(1, T, 1, n, k))
    nf.nf_expert_grad(dy, x, off, rows, 1, ws)
    a, b = dy[2:T - 1].double(), x[2:T - 1].double()
    close(rows[0, 1:1 + n * k].view(n, k), a.t() @ b, a.abs().t() @ b.abs(), T - 3)
    assert float(rows[0, 0]) == 7.0 and bool((rows[0, 1 + n * k:] == 7).all())
