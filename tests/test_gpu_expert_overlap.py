"""Results that lie between their operands' rows, in one buffer with them: taken, and equal to those in buffers of their
own."""
import pytest
import torch

import paper_2606_25759_amd as nf

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("W", [1, 2])
@pytest.mark.parametrize("n,k", [(24, 40), (23, 41), (1, 1)])
def test_product_between_rows(W, n, k):
    T, E = 30, 3
    g = torch.Generator().manual_seed(n)
    w = torch.randn(E, n, k, generator=g).bfloat16().to(DEV)
    off = torch.tensor([[0, 11, 11, 30]] * W, dtype=torch.int32, device=DEV)
    want = torch.zeros(W, T, n, dtype=torch.bfloat16, device=DEV)
    rows = torch.randn(W, T, k, generator=g).bfloat16().to(DEV)
    nf.nf_expert_product(rows, w, off, want)

    def check(x, y):
        x.copy_(rows)
        nf.nf_expert_product(x, w, off, y)
        assert torch.equal(y, want) and torch.equal(x, rows)

    both = torch.zeros(W, T, n + k, dtype=torch.bfloat16, device=DEV)
    check(both[..., :k], both[..., k:])
    check(both[..., n:], both[..., :n])
    both = torch.zeros(W, T, n + k + 5, dtype=torch.bfloat16, device=DEV)
    check(both[..., 3:3 + k], both[..., 3 + k:3 + k + n])
    # one whole behind the other, and between two rows of the other
    flat = torch.zeros(W * T * (n + k), dtype=torch.bfloat16, device=DEV)
    check(flat[:W * T * k].view(W, T, k), flat[W * T * k:].view(W, T, n))
    check(flat[W * T * n:].view(W, T, k), flat[:W * T * n].view(W, T, n))
    gap = W * T * max(n, k)
    flat = torch.zeros(W * T * (gap + max(n, k)), dtype=torch.bfloat16, device=DEV)
    ld = gap + max(n, k)
    check(flat.as_strided((W, T, k), (T * ld, ld, 1)), flat[7 * ld + k:7 * ld + k + W * T * n].view(W, T, n))
    check(flat[7 * ld + n:7 * ld + n + W * T * k].view(W, T, k), flat.as_strided((W, T, n), (T * ld, ld, 1)))
    check(flat.as_strided((W, T, k), (T * ld, ld, 1)), flat[k:].as_strided((W, T, n), (T * ld, ld, 1)))


def test_grad_behind_its_operands():
    T, E, n, k = 40, 2, 24, 40
    flat = torch.randn(T * (n + k) + E * n * k, device=DEV)
    dy, x, rows = flat[:T * n].view(T, n), flat[T * n:T * (n + k)].view(T, k), flat[T * (n + k):].view(1, -1)
    off = torch.tensor([0, 15, 40], dtype=torch.int32, device=DEV)
    ws = nf.empty_workspace(nf.nf_expert_grad_workspace_bytes(1, T, E, n, k))
    want = torch.empty(1, E * n * k, device=DEV)
    nf.nf_expert_grad(dy.clone(), x.clone(), off, want, 0, ws)
    nf.nf_expert_grad(dy, x, off, rows, 0, ws)
    assert torch.equal(rows, want)
