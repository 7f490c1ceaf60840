"""Matrices whose norm is far below eps: X is far below one, and its steps are nearly linear in it.

Tolerances as in test_gpu_orthogonal.py, relative to the result: 3e-3 of 11-bit operands, 2e-5 of 22-bit ones, and half
a unit of the result's type.  A batch holds norms from ten times eps to 1e-32 (times eps of 1e-7, X reaches 1e-25).
"""
import pytest
import torch

import paper_2606_25759_amd as nf
from tests.orthogonal_sizes import BF16, F32, SINGLE, SPLIT
from tests.test_gpu_orthogonal_tiles import BOUND, COEF, TORCH, UNIT, decaying, definition, off, workspace

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
NORMS = [1.0, 1e-6, 1e-7, 1e-8, 1e-9, 1e-10, 1e-11, 1e-12, 1e-13, 1e-15, 1e-20, 1e-32]


def of_norms(m, n, norms, seed, gauss=False):
    u = decaying(len(norms), m, n, 0, seed)
    if gauss:
        u.copy_(torch.randn(u.shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV))
    for k, norm in enumerate(norms):
        u[k] *= norm / torch.linalg.vector_norm(u[k].double())
    return u


@pytest.mark.parametrize("gauss", [False, True])
@pytest.mark.parametrize("m,n,products,dst_type", [
    (64, 576, SINGLE, F32), (7, 1, SPLIT, F32), (700, 40, SPLIT, BF16),      # a short side of one tile
    (130, 190, SINGLE, BF16), (130, 190, SPLIT, F32), (449, 385, SINGLE, F32),
    (769, 769, SINGLE, F32), (385, 385, SPLIT, F32),                         # larger tiles
    (100, 4000, SINGLE, BF16), (600, 385, SPLIT, BF16)])                     # steps at once by the Gram matrix
def test_norms(m, n, products, dst_type, gauss):
    u = of_norms(m, n, NORMS, m + n, gauss)
    d = torch.empty(u.shape, dtype=TORCH[dst_type], device=DEV)
    how = nf.orthogonal(products=products)
    nf.nf_orthogonalize(u, d, how, workspace(u, how))
    for k, norm in enumerate(NORMS):
        assert off(d[k], definition(u[k], [COEF] * 5)) <= BOUND[products] + UNIT[d.dtype], norm


@pytest.mark.parametrize("m,n", [(64, 576), (130, 190), (100, 4000)])
@pytest.mark.parametrize("triples", [
    [(1.5, -0.5, 0.0)] * 12,                                   # all of its steps below one
    [(0.1, 0.02, 0.0), (0.2, 0.1, 0.1), (3.0, -1.0, 0.5)],     # shrinks, then grows
    [(0.0, 1.5, 0.0), (0.0, 2.0, 1.0)],                        # no linear term
    [(-2.0, 1.0, 0.0), (1.875, -1.25, 0.375)]])
def test_coefficients(m, n, triples):
    norms = [1.0, 0.2, 1e-2, 1e-4]
    u = of_norms(m, n, norms, 5)
    d = torch.empty(u.shape, device=DEV)
    for products in (SINGLE, SPLIT):
        how = nf.orthogonal(products=products, steps=len(triples), coef=triples, eps=0.1)
        nf.nf_orthogonalize(u, d, how, workspace(u, how))
        for k, norm in enumerate(norms):
            want = definition(u[k], triples, eps=float(torch.tensor(0.1)))
            assert off(d[k], want) <= BOUND[products] + UNIT[d.dtype], (products, norm)


@pytest.mark.parametrize("weight,products", [(torch.float32, SPLIT), (torch.bfloat16, SINGLE)])
@pytest.mark.parametrize("m,n", [(64, 576), (449, 385)])
def test_update(m, n, weight, products):
    """Weights that begin at zero are the update alone."""
    norms = [1.0, 1e-9, 1e-12, 1e-15]
    u = of_norms(m, n, norms, 3)
    mom, w = torch.zeros(u.shape, device=DEV), torch.zeros(u.shape, dtype=weight, device=DEV)
    how = nf.orthogonal(products=products)
    nf.nf_orthogonal_update(u, mom, w, nf.matrix_step(0.02, 0.9, False, 0.1, 1.5), how, workspace(u, how))
    for k, norm in enumerate(norms):
        want = -0.02 * 1.5 * definition(u[k], [COEF] * 5)
        assert off(w[k], want) <= BOUND[products] + UNIT[weight] + 4 * UNIT[torch.float32], norm


def test_the_others_of_a_batch_keep_their_bits():
    u = of_norms(130, 190, [1.0, 1e-12, 1.0, 0.0], 2)
    how = nf.orthogonal()
    d, alone = torch.empty(u.shape, device=DEV), torch.empty(1, 130, 190, device=DEV)
    nf.nf_orthogonalize(u, d, how, workspace(u, how))
    for k in range(3):
        nf.nf_orthogonalize(u[k:k + 1], alone, how, workspace(u[k:k + 1], how))
        assert torch.equal(alone[0], d[k])
    assert bool((d[3] == 0).all())
