"""nf_grad_norm, nf_grad_clip and nf_grad_norm_clip against sums in 64 bits.

A norm's FP64 sum of n squares is off by less than n 2^-53 of it, nothing
beside the rounding to FP32 (half a step: 2^-24).  The factor and the scaled
tensors follow from the norm that was returned by operations that round once
each, so they have equal bits.
"""
import numpy as np
import pytest
import torch

import paper_2606_25759_amd as nf

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def norm_of(tensors):
    return float(torch.stack([t.double().square().sum() for t in tensors]).sum().sqrt()) if tensors else 0.0


def factor(norm, max_norm, eps=1e-6):
    """The factor by a norm that the library returned."""
    below = np.float64(np.float32(norm)) + np.float64(np.float32(eps))
    with np.errstate(all="ignore"):
        ratio = np.float64(1.0) if below == 0 else np.float64(np.float32(max_norm)) / below
    return np.float32(1.0) if ratio >= 1 else np.float32(ratio)


def same(a, b):
    return torch.equal(torch.nan_to_num(a.float(), nan=12345.0), torch.nan_to_num(b.float(), nan=12345.0))


def check(src, dst, groups, n_groups, max_norm):
    """Norms, then clipping by them, then both in one call: the norms by the definition, the rest bit for bit."""
    before = [t.clone() for t in src]
    plan = nf.norm_plan(src, dst, groups, n_groups)
    ws = nf.empty_workspace(nf.nf_grad_norm_workspace_bytes(plan))
    ws.fill_(0xFF)
    norms = torch.full((n_groups,), -1.0, device=DEV)
    nf.nf_grad_norm(plan, norms, ws)
    got = norms.cpu().numpy()
    for g in range(n_groups):
        want = norm_of([t for t, k in zip(before, groups) if k == g])
        assert abs(got[g] - want) <= 1.001 * 2.0 ** -24 * want + 2.0 ** -149, (g, got[g], want)
    if dst is None:
        return
    by = [torch.tensor(factor(n, max_norm), device=DEV) for n in got]
    want = [(t.float() * by[k]).to(d.dtype) for t, d, k in zip(before, dst, groups)]
    nf.nf_grad_clip(plan, norms, max_norm)
    assert all(same(d, w) for d, w in zip(dst, want))
    for t, b in zip(src, before):
        t.copy_(b)
    again = torch.full((n_groups,), -1.0, device=DEV)
    ws.fill_(0x7F)
    nf.nf_grad_norm_clip(plan, max_norm, again, ws)
    assert torch.equal(again, norms)
    assert all(same(d, w) for d, w in zip(dst, want))


SIZES = {"one": [1], "odd": [1, 2, 3, 7, 8, 9, 63, 64, 65, 511, 513, 1023, 1025], "empty": [0, 5, 0],
         "nothing": [], "large": [1_000_003, 4, 300_000], "many": [(i * 37) % 5000 + 1 for i in range(700)],
         "block": [32_768, 31_744, 1024]}


@pytest.mark.parametrize("to", ["none", "f32", "bf16", "f16", "same"])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("sizes", list(SIZES))
def test_sizes(sizes, kind, to):
    g = torch.Generator().manual_seed(len(SIZES[sizes]))
    n = SIZES[sizes]
    flat = torch.randn(sum(n) + 1, generator=g).to(TYPES[kind]).to(DEV)
    src = list(flat[1:].split(n)) if n else []  # one after the other, no alignment
    groups = [i % 3 for i in range(len(n))]
    if to == "none":
        dst = None
    elif to == "same":
        dst = src
    else:
        around = torch.full((sum(n) + 2,), 5.0, dtype=TYPES[to], device=DEV)
        dst = list(around[1:-1].split(n)) if n else []
    check(src, dst, groups, 4, 0.3)  # the last group has no tensor
    if to not in ("none", "same"):
        assert float(around[0]) == 5.0 and float(around[-1]) == 5.0


@pytest.mark.parametrize("kind", list(TYPES))
def test_strides(kind):
    """Rows apart, transposed, slices of three dimensions, parts of one buffer between one another's rows."""
    g = torch.Generator().manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g).to(TYPES[kind]).to(DEV)  # noqa: E731
    a, b, c = rand(300, 70), rand(40, 5000), rand(6, 33, 50)
    src = [a[:, :31], a[:, 31:33], a[:, 33:], b.t(), c[:, 3:20, 1:], c[:, :3, :], rand(3, 40_000)[:, :39_999],
           rand(50, 4)[::2, 1], rand(7, 1)[:, 0], rand(2, 3, 4).permute(2, 0, 1)]
    rows = torch.full((sum(t.numel() for t in src) + 3,), 2.0, device=DEV)
    at, places = 1, []
    for t in src:
        places.append(rows[at:at + t.numel()].view(t.shape))
        at += t.numel()
    check(src, places, [0, 1] * 5, 2, 1.7)
    assert float(rows[0]) == 2.0 and bool((rows[-2:] == 2.0).all())
    before = [t.clone() for t in (a, b, c)]
    check(src, src, [1, 0] * 5, 2, 1.7)  # in place
    outside = torch.ones_like(c, dtype=torch.bool)
    outside[:, 3:20, 1:] = False
    outside[:, :3, :] = False
    assert torch.equal(c[outside], before[2][outside])


@pytest.mark.parametrize("kind", list(TYPES))
def test_infinities_nan_and_scales(kind):
    tiny, big = torch.finfo(TYPES[kind]).tiny, torch.finfo(TYPES[kind]).max
    make = lambda v: torch.full((1500,), v, dtype=TYPES[kind], device=DEV)  # noqa: E731
    src = [make(1.0), make(1.0), make(0.0), make(tiny), make(big / 64)]
    src[0][700] = float("inf")
    src[1][3] = float("nan")
    dst = [torch.empty(1500, device=DEV) for _ in src]
    plan = nf.norm_plan(src, dst, range(5))
    norms, ws = torch.empty(5, device=DEV), nf.empty_workspace(nf.nf_grad_norm_workspace_bytes(plan))
    nf.nf_grad_norm_clip(plan, 2.0, norms, ws)
    n = norms.cpu().numpy()
    assert np.isposinf(n[0]) and np.isnan(n[1]) and n[2] == 0
    for i in (3, 4):
        assert abs(n[i] - norm_of([src[i]])) <= 1.001 * 2.0 ** -24 * norm_of([src[i]]) + 2.0 ** -149
    assert bool(dst[0][700].isnan()) and int((dst[0] == 0).sum()) == 1499
    assert bool(dst[1].isnan().all()) and bool((dst[2] == 0).all())
    assert torch.equal(dst[3], src[3].float())  # nothing to clip
    assert torch.equal(dst[4], src[4].float() * torch.tensor(factor(n[4], 2.0), device=DEV))
    # nothing below the line: the factor is one, whatever max_norm
    nf.nf_grad_clip(nf.norm_plan(src[2:3], dst[2:3]), torch.zeros(1, device=DEV), 0.0, eps=0.0)
    assert bool((dst[2] == 0).all())
    nf.nf_grad_clip(nf.norm_plan(src[3:4], dst[3:4]), torch.ones(1, device=DEV), 0.0)
    assert bool((dst[3] == 0).all())


def test_in_place_below_the_limit_keeps_bits():
    t = torch.randn(5000, device=DEV).bfloat16()
    t[3] = -0.0
    before = t.clone()
    plan = nf.norm_plan([t], [t])
    norms, ws = torch.empty(1, device=DEV), nf.empty_workspace(nf.nf_grad_norm_workspace_bytes(plan))
    nf.nf_grad_norm_clip(plan, 1e6, norms, ws)
    assert torch.equal(t.view(torch.int16), before.view(torch.int16))


def test_a_tensor_read_twice_counts_twice():
    t = torch.randn(3000, device=DEV)
    norms = torch.empty(1, device=DEV)
    plan = nf.norm_plan([t, t, t[5:50]])
    nf.nf_grad_norm(plan, norms, nf.empty_workspace(nf.nf_grad_norm_workspace_bytes(plan)))
    want = norm_of([t, t, t[5:50]])
    assert abs(float(norms) - want) <= 1.001 * 2.0 ** -24 * want


def test_far_elements():
    """Elements past 2^31 of a row."""
    n = 2 ** 31 + 5000
    row = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    row[-1], row[0], row[2 ** 31 + 7] = 3.0, 4.0, 12.0
    norms = torch.empty(1, device=DEV)
    plan = nf.norm_plan([row], [row])
    nf.nf_grad_norm_clip(plan, 1.3, norms, nf.empty_workspace(nf.nf_grad_norm_workspace_bytes(plan)), eps=0.0)
    assert float(norms) == 13.0
    by = torch.tensor(factor(13.0, 1.3, 0.0), device=DEV)
    for at, v in ((-1, 3.0), (0, 4.0), (2 ** 31 + 7, 12.0)):
        assert float(row[at]) == float((v * by).bfloat16())


def test_other_stream_and_graph_replays():
    """Two graphs that share a workspace, replayed one after the other with new values and eager calls between."""
    a, b = torch.empty(3, 70_001, device=DEV), torch.empty(900, device=DEV, dtype=torch.float16)
    rows = torch.empty(2, 300_000, device=DEV)
    plans = [nf.norm_plan([a], [rows[0, :210_003].view(3, -1)]), nf.norm_plan([b, a[1]], [rows[1, :900], rows[1, 901:70_902]], [1, 0])]
    ws = nf.empty_workspace(max(nf.nf_grad_norm_workspace_bytes(p) for p in plans))
    norms = [torch.empty(p.plan.groups, device=DEV) for p in plans]

    def fill(seed):
        g = torch.Generator().manual_seed(seed)
        a.copy_(torch.randn(a.shape, generator=g) * 10 ** seed)
        b.copy_(torch.randn(b.shape, generator=g))

    def calls(i):
        nf.nf_grad_norm_clip(plans[i], 2.5, norms[i], ws)

    fill(0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for i in range(2):
            calls(i)
    side.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in plans]
    for i in range(2):
        with torch.cuda.graph(graphs[i]):
            calls(i)
    for seed in range(4):
        fill(seed)
        rows.fill_(7.0)
        for i in range(2):
            calls(i)
        torch.cuda.synchronize()
        want = [t.clone() for t in (rows, *norms)]
        rows.fill_(7.0)
        for t in norms:
            t.fill_(-1.0)
        for i in range(2):
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, w) for x, w in zip((rows, *norms), want))
