"""Every product kernel of the orthogonalisation against the definition in 64 bits.

Tolerances as in test_gpu_orthogonal.py (2-norm of the difference over 2-norm
of the result): 11-bit operands 3e-3 and 22-bit ones 2e-5 at up to five steps,
each plus half a unit of the result's type.
"""
import numpy as np
import pytest
import torch

import paper_2606_25759_amd as nf
from tests.orthogonal_sizes import BF16, SINGLE, SIZES, SPLIT, kernels_of

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
COEF = (3.4445, -4.7750, 2.0315)
BOUND = {SINGLE: 3e-3, SPLIT: 2e-5}
TORCH = {BF16: torch.bfloat16, nf.NF_TYPE_F32: torch.float32}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -9}


def definition(u, triples, eps=1e-7):
    """One matrix, in 64 bits."""
    x = u.double()
    x = x / (torch.linalg.vector_norm(x) + eps)
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    for a, b, c in triples:
        s = x @ x.t().contiguous()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.t() if tall else x


def decaying(batch, m, n, gap, seed):
    """Matrices `gap` elements apart, rows 3: NaN between them."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = max(1, min(m, n) // 8)
    s = torch.logspace(0, -2, r, device=DEV)
    flat = torch.full((batch * (m * (n + 3) + gap),), float("nan"), device=DEV)
    u = flat.as_strided((batch, m, n), (m * (n + 3) + gap, n + 3, 1))
    for k in range(batch):
        left = torch.randn(m, r, generator=g, device=DEV) * s
        u[k] = 1e-3 * (left @ torch.randn(r, n, generator=g, device=DEV)
                       + 0.01 * r ** 0.5 * torch.randn(m, n, generator=g, device=DEV))
    return u


def workspace(u, how):
    ws = nf.empty_workspace(nf.nf_orthogonal_workspace_bytes(u.shape[1], u.shape[2], u.shape[0], how))
    ws.fill_(0xFF)
    return ws


def off(got, want):
    return float(torch.linalg.vector_norm(got.double() - want) / torch.linalg.vector_norm(want))


@pytest.mark.parametrize("batch,m,n,products,dst_type", SIZES)
def test_every_kernel(batch, m, n, products, dst_type):
    u = decaying(batch, m, n, 5, m + n)
    out = torch.full((batch * (m * (n + 5) + 7),), 7.0, dtype=TORCH[dst_type], device=DEV)
    d = out.as_strided((batch, m, n), (m * (n + 5) + 7, n + 5, 1))
    how = nf.orthogonal(products=products)
    nf.nf_orthogonalize(u, d, how, workspace(u, how))
    for k in range(batch):
        assert off(d[k], definition(u[k], [COEF] * 5)) <= BOUND[products] + UNIT[d.dtype], k
    inside = torch.zeros(out.shape, dtype=torch.bool, device=DEV)
    inside.as_strided(d.shape, d.stride()).fill_(True)
    assert bool((out[~inside] == 7.0).all())
    again = torch.empty(batch, m, n, dtype=d.dtype, device=DEV)
    nf.nf_orthogonalize(u, again, how, workspace(u, how))
    assert torch.equal(again, d)


@pytest.mark.parametrize("batch,m,n,products,dst_type", [s for s in SIZES if min(s[1:3]) > 64 and s[0] <= 16])
@pytest.mark.parametrize("steps", [1, 2, 4])
def test_steps(steps, batch, m, n, products, dst_type):
    """Another triple for every step, and both places that X's transpose can end up in."""
    triples = [COEF, (2.0, -1.5, 0.5), (1.5, -0.5, 0.0), (1.875, -1.25, 0.375)][-steps:]
    u = decaying(batch, m, n, 0, m + n + steps)
    d = torch.empty(batch, m, n, dtype=TORCH[dst_type], device=DEV)
    how = nf.orthogonal(products=products, steps=steps, coef=triples)
    nf.nf_orthogonalize(u, d, how, workspace(u, how))
    for k in (0, batch - 1):
        assert off(d[k], definition(u[k], triples)) <= BOUND[products] + UNIT[d.dtype], k


# An emulation in NumPy of the roundings of 11-bit operands (Gaussian matrices of 128 x 300, 512 x 512 and 200 x 900)
# is off by at most 1.9e-3 after seven steps of the default coefficients, 3.4e-3 after twelve, and 5.1e-4 after twelve
# of coefficients that converge: half as much again is allowed.  22 bits: what nf.h says, and as much again.
@pytest.mark.parametrize("gauss", [False, True])
@pytest.mark.parametrize("coef,steps,bound", [
    (COEF, 7, {SINGLE: 2.9e-3, SPLIT: 6e-5}), (COEF, 8, {SINGLE: 5.1e-3, SPLIT: 6e-5}),
    (COEF, 12, {SINGLE: 5.1e-3, SPLIT: 6e-5}), ((2.0, -1.5, 0.5), 12, {SINGLE: 7.7e-4, SPLIT: 6e-5}),
    ((1.5, -0.5, 0.0), 11, {SINGLE: 7.7e-4, SPLIT: 6e-5})])
@pytest.mark.parametrize("batch,m,n", [(2, 190, 130), (1, 512, 512), (30, 449, 385), (16, 769, 769)])
def test_many_steps(batch, m, n, coef, steps, bound, gauss):
    """Steps one by one, the rounding of every one of them in the result."""
    u = decaying(batch, m, n, 0, m + n + steps)
    if gauss:
        u.copy_(torch.randn(u.shape, generator=torch.Generator(device=DEV).manual_seed(steps), device=DEV))
    d = torch.empty(batch, m, n, device=DEV)
    for products in (SINGLE, SPLIT):
        how = nf.orthogonal(products=products, steps=steps, coef=coef)
        assert nf.nf_orthogonal_path(m, n, batch, how, nf.NF_TYPE_F32).rounds == steps
        nf.nf_orthogonalize(u, d, how, workspace(u, how))
        for k in (0, batch - 1):
            assert off(d[k], definition(u[k], [coef] * steps)) <= bound[products], (products, k)


@pytest.mark.parametrize("batch,m,n", [(30, 449, 385), (16, 769, 769), (8, 500, 4000), (8, 4000, 500)])
def test_nan_stays_in_its_matrix(batch, m, n):
    u = decaying(batch, m, n, 0, 1)
    how = nf.orthogonal()
    want, got = (torch.empty(batch, m, n, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    nf.nf_orthogonalize(u, want, how, workspace(u, how))
    u[1, m - 1, n - 1] = float("nan")
    u[2, 0, 0] = float("inf")
    u[3] = 0.0
    nf.nf_orthogonalize(u, got, how, workspace(u, how))
    assert bool(got[1:3].isnan().all()) and bool((got[3] == 0).all())
    assert torch.equal(got[4:], want[4:]) and torch.equal(got[0], want[0])


@pytest.mark.parametrize("weight,products", [(torch.bfloat16, SINGLE), (torch.float32, SPLIT), (torch.float32, SINGLE)])
@pytest.mark.parametrize("batch,m,n", [(30, 449, 385), (16, 769, 769), (8, 500, 4000), (8, 600, 385), (40, 257, 449)])
def test_update(batch, m, n, weight, products):
    """w = (1 - lr wd) w - lr scale O(g + mu M) by the large tiles; its error is at most lr scale times O's."""
    lr, mu, decay, scale = 0.02, 0.9, 0.1, 1.5
    g = torch.Generator(device=DEV).manual_seed(m)
    u = decaying(batch, m, n, 9, n)
    mom = torch.randn(batch, m, n + 2, generator=g, device=DEV)[:, :, 1:-1] * 1e-3
    w = (torch.randn(batch, m, n + 1, generator=g, device=DEV) * 0.02).to(weight)[:, :, 1:]
    m64, w64 = mom.double(), w.double()
    how = nf.orthogonal(products=products)
    nf.nf_orthogonal_update(u, mom, w, nf.matrix_step(lr, mu, True, decay, scale), how, workspace(u, how))
    m64 = float(np.float32(mu)) * m64 + u.double()
    assert off(mom, m64) <= 2 * UNIT[torch.float32]
    x = u.double() + mu * m64
    for k in range(batch):
        o = definition(x[k], [COEF] * 5)
        want = (1 - lr * decay) * w64[k] - lr * scale * o
        slack = lr * scale * BOUND[products] * float(torch.linalg.vector_norm(o) / torch.linalg.vector_norm(want))
        assert off(w[k], want) <= UNIT[weight] + 4 * UNIT[torch.float32] + slack, k


def test_other_stream_and_replays():
    """Tiles of 256, 128 and 64 with a shared k in one call: on a side stream, and replayed."""
    batch, m, n = 8, 500, 4000
    assert {t for t, _, _, _ in kernels_of(batch, m, n, SINGLE, BF16)} == {64, 128, 256}
    u = decaying(batch, m, n, 0, 2)
    how = nf.orthogonal()
    ws = workspace(u, how)
    dst, want = (torch.empty(batch, m, n, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        nf.nf_orthogonalize(u, dst, how, ws)
    side.synchronize()
    nf.nf_orthogonalize(u, want, how, ws)
    assert torch.equal(dst, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nf.nf_orthogonalize(u, dst, how, ws)
    for k in range(3):
        u.copy_(decaying(batch, m, n, 0, 10 + k))
        nf.nf_orthogonalize(u, want, how, workspace(u, how))
        dst.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dst, want)
