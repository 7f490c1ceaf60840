"""nf_orthogonalize and nf_orthogonal_update against the definition in 64 bits.

Tolerances (2-norm of the difference over 2-norm of the result).  Products of
11-bit operands: each of A, B and X is rounded once a step with a relative
error of 2^-12 at most a value, and a step multiplies what is there by less
than the largest of |a|, |a + 3b s^2 + 5c s^4| only in directions that
rounding does not reach; an emulation of the same roundings on these kinds of
inputs stays below 1.5e-3, so 3e-3 (plus half a unit of the result's type).
Products of 22-bit operands: FP32 sums are what is left, 2e-5 for spectra that
decay to 1e-2, and 2e-4 where nearly all is in one direction, which a^5 = 485
sets apart from the noise below it.
"""
import numpy as np
import pytest
import torch

import paper_2606_25759_amd as nf

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
COEF = (3.4445, -4.7750, 2.0315)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -9, "f16": 2.0 ** -12}
BOUND = {nf.NF_PRODUCTS_SINGLE: {"gauss": 3e-3, "decay": 3e-3, "rank1": 3e-3},
         nf.NF_PRODUCTS_SPLIT: {"gauss": 2e-5, "decay": 2e-5, "rank1": 2e-4}}
BOTH = [nf.NF_PRODUCTS_SINGLE, nf.NF_PRODUCTS_SPLIT]


def make(kind, m, n, seed, batch=None):
    g = np.random.default_rng(seed)
    if batch is not None:
        return np.stack([make(kind, m, n, seed + 100 * k) for k in range(batch)])
    if kind == "gauss":
        x = g.standard_normal((m, n))
    elif kind == "decay":
        r = max(1, min(m, n) // 8)
        x = (g.standard_normal((m, r)) * np.logspace(0, -2, r)) @ g.standard_normal((r, n))
        x = x + 0.01 * r ** 0.5 * g.standard_normal((m, n))
    else:
        x = g.standard_normal((m, 1)) @ g.standard_normal((1, n)) + 1e-4 * g.standard_normal((m, n))
    return x * 1e-3


def exact(u, steps=5, coef=COEF, eps=1e-7):
    """The definition, by the singular values: each step maps s to a s + b s^3 + c s^5."""
    u = np.asarray(u, np.float64)
    p, s, q = np.linalg.svd(u, full_matrices=False)
    s = s / (np.linalg.norm(u) + eps) if np.linalg.norm(u) else s
    for k in range(steps):
        a, b, c = coef if np.ndim(coef) == 1 else coef[k]
        s = a * s + b * s ** 3 + c * s ** 5
    return (p * s) @ q


def workspace(t, how):
    b = t.shape[0] if t.dim() == 3 else 1
    need = nf.nf_orthogonal_workspace_bytes(t.shape[-2], t.shape[-1], b, how)
    ws = nf.empty_workspace(need)
    ws.fill_(0xFF)  # NaN to every type: nothing left there may matter
    return ws


def far(got, want):
    got = got.double().cpu().numpy()
    n = np.linalg.norm(want)
    return np.linalg.norm(got - want) / (n if n else 1.0)


SHAPES = [(1, 1), (1, 7), (7, 1), (2, 2), (3, 200), (63, 65), (64, 64), (65, 64), (64, 577), (128, 128), (129, 257),
          (300, 100), (257, 511), (512, 256), (700, 333)]


@pytest.mark.parametrize("products", BOTH)
@pytest.mark.parametrize("kind", ["gauss", "decay"])
@pytest.mark.parametrize("m,n", SHAPES)
def test_shapes(m, n, kind, products):
    u = torch.from_numpy(make(kind, m, n, m * 1000 + n)).float().to(DEV)
    dst = torch.full((m, n), float("nan"), device=DEV)
    how = nf.orthogonal(products=products)
    nf.nf_orthogonalize(u, dst, how, workspace(u, how))
    assert far(dst, exact(u.cpu().numpy())) <= BOUND[products][kind] + UNIT["f32"]


@pytest.mark.parametrize("products", BOTH)
@pytest.mark.parametrize("m,n", [(96, 160), (260, 130)])
def test_one_large_direction(m, n, products):
    u = torch.from_numpy(make("rank1", m, n, 5)).float().to(DEV)
    dst = torch.empty_like(u)
    how = nf.orthogonal(products=products)
    nf.nf_orthogonalize(u, dst, how, workspace(u, how))
    assert far(dst, exact(u.cpu().numpy())) <= BOUND[products]["rank1"]


@pytest.mark.parametrize("products", BOTH)
@pytest.mark.parametrize("src", list(TYPES))
@pytest.mark.parametrize("dst", list(TYPES))
def test_types_strides_and_surroundings(src, dst, products):
    """Rows and matrices apart, and nothing written between them."""
    for batch, m, n in ((3, 70, 45), (2, 33, 130)):
        u = torch.from_numpy(make("decay", m, n, 9, batch)).to(DEV).to(TYPES[src])
        flat = torch.full((batch * (m * (n + 5) + 11),), float("nan"), dtype=TYPES[src], device=DEV)
        s = flat.as_strided((batch, m, n), (m * (n + 5) + 11, n + 5, 1))
        s.copy_(u)
        out = torch.full((batch * (m * (n + 3) + 7),), 7.0, dtype=TYPES[dst], device=DEV)
        d = out.as_strided((batch, m, n), (m * (n + 3) + 7, n + 3, 1))
        how = nf.orthogonal(products=products)
        nf.nf_orthogonalize(s, d, how, workspace(s, how))
        for k in range(batch):
            want = exact(u[k].double().cpu().numpy())
            assert far(d[k], want) <= BOUND[products]["decay"] + UNIT[dst]
        inside = torch.zeros(out.shape, dtype=torch.bool, device=DEV)
        inside.as_strided(d.shape, d.stride()).fill_(True)
        assert bool((out[~inside] == 7.0).all())


@pytest.mark.parametrize("products", BOTH)
def test_zeros_nan_and_scale(products):
    """A zero matrix gives zeros, one with a NaN or an infinity NaN everywhere, the others of the batch
    are what they are alone; no scale of FP32 overflows or vanishes."""
    m, n = 70, 90
    u = make("gauss", m, n, 3, 6)
    u[1] = 0.0
    u[2, 5, 6] = np.nan
    u[3, 69, 89] = np.inf
    u[4] *= 1e-30
    u[5] *= 1e36
    t = torch.from_numpy(u).float().to(DEV)
    dst = torch.empty_like(t)
    how = nf.orthogonal(products=products, eps=0.0)
    nf.nf_orthogonalize(t, dst, how, workspace(t, how))
    assert bool((dst[1] == 0).all())
    assert bool(dst[2].isnan().all()) and bool(dst[3].isnan().all())
    for k in (0, 4, 5):
        assert far(dst[k], exact(t[k].cpu().numpy(), eps=0.0)) <= BOUND[products]["gauss"]
    alone = torch.empty_like(t[0])
    nf.nf_orthogonalize(t[0], alone, how, workspace(t[0], how))
    assert torch.equal(alone, dst[0])


@pytest.mark.parametrize("products", BOTH)
@pytest.mark.parametrize("coef", [COEF, (1.5, -0.5, 0.0), (2.0, -1.5, 0.5)])
@pytest.mark.parametrize("steps", [1, 2, 12])
def test_steps_and_coefficients(steps, coef, products):
    """Also a triple for every step: the last one another."""
    m, n = 60, 130
    u = torch.from_numpy(make("gauss", m, n, 8)).float().to(DEV)
    triples = [coef] * (steps - 1) + [(1.875, -1.25, 0.375)]
    how = nf.orthogonal(products=products, steps=steps, coef=triples, eps=0.01)
    dst = torch.empty_like(u)
    nf.nf_orthogonalize(u, dst, how, workspace(u, how))
    assert far(dst, exact(u.cpu().numpy(), steps, triples, eps=np.float32(0.01))) <= BOUND[products]["gauss"]


@pytest.mark.parametrize("dst", ["bf16", "f32"])
@pytest.mark.parametrize("products", BOTH)
@pytest.mark.parametrize("kind", ["gauss", "decay"])
@pytest.mark.parametrize("batch,m,n", [(12, 100, 4000), (3, 6001, 150), (1, 64, 20_000), (30, 30, 2000),
                                       (2, 300, 5000)])
def test_long_sides(batch, m, n, kind, products, dst):
    """Where several steps are taken at once by the Gram matrix, and a tile's k by several blocks."""
    u = torch.from_numpy(make(kind, m, n, m + n, batch)).float().to(DEV)
    d = torch.empty(u.shape, dtype=TYPES[dst], device=DEV)
    how = nf.orthogonal(products=products)
    nf.nf_orthogonalize(u, d, how, workspace(u, how))
    for k in range(0, batch, 5):
        assert far(d[k], exact(u[k].cpu().numpy())) <= BOUND[products][kind] + UNIT[dst]


@pytest.mark.parametrize("coef", [COEF, (1.5, -0.5, 0.0), (2.0, -1.5, 0.5), (3.0, -3.2, 1.2)])
@pytest.mark.parametrize("steps", [1, 2, 4, 7, 12])
@pytest.mark.parametrize("batch,m,n", [(12, 100, 4000), (2, 40, 900)])
def test_long_sides_steps(batch, m, n, steps, coef):
    u = torch.from_numpy(make("gauss", m, n, 3, batch)).float().to(DEV)
    d = torch.empty(u.shape, dtype=torch.bfloat16, device=DEV)
    triples = [coef] * (steps - 1) + [(1.875, -1.25, 0.375)]
    how = nf.orthogonal(steps=steps, coef=triples)
    nf.nf_orthogonalize(u, d, how, workspace(u, how))
    for k in (0, batch - 1):
        want = exact(u[k].cpu().numpy(), steps, triples)
        assert far(d[k], want) <= BOUND[nf.NF_PRODUCTS_SINGLE]["gauss"] + UNIT["bf16"]


def test_in_place_other_stream_and_repeatable():
    u = torch.from_numpy(make("decay", 200, 150, 1, 2)).float().to(DEV)
    how = nf.orthogonal()
    ws = workspace(u, how)
    a, b = torch.empty_like(u), u.clone()
    nf.nf_orthogonalize(u, a, how, ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        nf.nf_orthogonalize(b, b, how, ws)
    side.synchronize()
    assert torch.equal(a, b)


def test_graph_replays():
    u = torch.from_numpy(make("decay", 130, 150, 2)).float().to(DEV)
    how = nf.orthogonal()
    ws, dst, want = workspace(u, how), torch.empty_like(u), torch.empty_like(u)
    nf.nf_orthogonalize(u, dst, how, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        nf.nf_orthogonalize(u, dst, how, ws)
    for k in range(4):
        u.copy_(torch.from_numpy(make("gauss", 130, 150, 20 + k)).float())
        nf.nf_orthogonalize(u, want, how, workspace(u, how))
        dst.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(dst, want)


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("grad", list(TYPES))
@pytest.mark.parametrize("weight", list(TYPES))
def test_update(weight, grad, nesterov):
    """Three steps: M = mu M + g, U = g + mu M or M, w = (1 - lr wd) w - lr scale O."""
    for batch, m, n in ((2, 90, 40), (1, 130, 190)):
        products = nf.NF_PRODUCTS_SINGLE if weight == "bf16" else nf.NF_PRODUCTS_SPLIT
        how = nf.orthogonal(products=products)
        step = nf.matrix_step(lr=0.02, momentum=0.9, nesterov=nesterov, weight_decay=0.1, scale=1.5)
        g = np.random.default_rng(4)
        mom = torch.from_numpy(g.standard_normal((batch, m, n + 3)) * 1e-3).float().to(DEV)[:, :, :n]
        w = torch.from_numpy(g.standard_normal((batch, m, n + 1)) * 0.02).to(DEV).to(TYPES[weight])[:, :, 1:]
        for k in range(3):
            u = torch.from_numpy(make("decay", m, n, 50 + k, batch)).to(DEV).to(TYPES[grad])
            g64, m64, w64 = (t.double().cpu().numpy() for t in (u, mom, w))
            nf.nf_orthogonal_update(u, mom, w, step, how, workspace(u, how))
            m64 = np.float64(np.float32(0.9)) * m64 + g64
            # two roundings of M, and one more of U
            assert far(mom, m64) <= 2 * UNIT["f32"]
            x = g64 + 0.9 * m64 if nesterov else m64
            o = np.stack([exact(x[b]) for b in range(batch)])
            want = (1 - 0.02 * 0.1) * w64 - 0.02 * 1.5 * o
            slack = 0.03 * BOUND[products]["decay"] * np.linalg.norm(o) / np.linalg.norm(want)
            assert far(w, want) <= UNIT[weight] + 4 * UNIT["f32"] + slack


def test_empty():
    how = nf.orthogonal()
    ws = nf.empty_workspace(256)
    for shape in ((0, 5), (5, 0), (0, 4, 4), (2, 0, 3)):
        t = torch.empty(shape, device=DEV)
        nf.nf_orthogonalize(t, torch.empty_like(t), how, ws)
        nf.nf_orthogonal_update(t, torch.empty_like(t), torch.empty_like(t), nf.matrix_step(0.1), how, ws)
    torch.cuda.synchronize()
