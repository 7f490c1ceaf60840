"""nf_embedding_lookup and nf_embedding_grad against plain implementations.

The lookup is one FP32 product rounded once: equal bits.  A row of the
gradient is an FP32 sum of n terms in some order, times the scale: its error
is at most (n + 3) 2^-24 times the sum of the terms' absolute values (times
the scale; with what was there before counted as a term).
"""
import numpy as np
import pytest
import torch

import paper_2606_25759_amd as nf

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.mark.parametrize("table", list(TYPES))
@pytest.mark.parametrize("out", list(TYPES))
def test_lookup(table, out):
    g = torch.Generator().manual_seed(1)
    for V, d, T, pad in ((50, 64, 1, 0), (7, 1, 130, 0), (100, 515, 33, 3), (1000, 1024, 257, 0), (33, 8, 0, 0),
                         (12, 2056, 19, 8), (5, 24, 1000, 4)):
        t = torch.randn(V, d + pad, generator=g).to(TYPES[table])[:, :d].to(DEV)
        big = torch.randn(V, d + pad, generator=g).to(TYPES[table]).to(DEV)
        t = big[:, :d]  # rows apart
        for kind in (torch.int32, torch.int64):
            ids = torch.randint(-3, V + 3, (T,), generator=g).to(kind).to(DEV)
            buf = torch.full((T, d + pad), 5.0, dtype=TYPES[out], device=DEV)
            nf.nf_embedding_lookup(t, ids, buf[:, :d], scale=1.7)
            ok = (ids >= 0) & (ids < V)
            want = t[ids.long().clamp(0, V - 1)].float() * torch.tensor(1.7, device=DEV)
            want = torch.where(ok[:, None], want, torch.zeros_like(want)).to(TYPES[out])
            assert torch.equal(buf[:, :d], want)
            assert bool((buf[:, d:] == 5.0).all())


def test_lookup_far_ids():
    """Ids beyond 32 bits are outside every table; infinities and NaN in the table stay what they are."""
    t = torch.tensor([[1.0, float("inf")], [float("nan"), -2.0]], device=DEV)
    ids = torch.tensor([2 ** 32, -2 ** 32, 2 ** 32 + 1, 0, 1, 2 ** 63 - 1, -2 ** 63], device=DEV)
    out = torch.full((7, 2), 9.0, device=DEV)
    nf.nf_embedding_lookup(t, ids, out, scale=2.0)
    o = out.cpu().numpy()
    assert np.array_equal(o[[0, 1, 2, 5, 6]], np.zeros((5, 2), np.float32))
    assert o[3, 0] == 2.0 and np.isposinf(o[3, 1]) and np.isnan(o[4, 0]) and o[4, 1] == -4.0


def check_grad(W, T, V, d, dy_type="f32", ids=None, kind=torch.int64, lead=0, extra=0, accumulate=False, padding=-1,
               scale=1.25, seed=0):
    g = torch.Generator().manual_seed(seed)
    big = torch.randn(W, T, d + extra, generator=g).to(TYPES[dy_type]).to(DEV)
    dy = big[:, :, :d]
    if ids is None:
        ids = torch.randint(0, V, (W, T), generator=g)
    ids = ids.to(kind).to(DEV)
    stride = (lead + V * d + 8) // 4 * 4
    rows = torch.randn(W, stride, generator=g).to(DEV)
    before = rows.clone()
    ws = nf.empty_workspace(nf.nf_embedding_workspace_bytes(W, T, V, d))
    ws.fill_(0xFF)
    nf.nf_embedding_grad(dy, ids, rows, lead, V, ws, scale=scale, padding_id=padding, accumulate=accumulate)
    seg = slice(lead, lead + V * d)
    outside = torch.ones(stride, dtype=torch.bool)
    outside[seg] = False
    assert torch.equal(rows[:, outside.to(DEV)], before[:, outside.to(DEV)])
    for w in range(W):
        i = ids[w].cpu().long()
        ok = (i >= 0) & (i < V) & (i != padding)
        i, x = i[ok], dy[w].cpu().double()[ok] * float(np.float32(scale))
        total, size = torch.zeros(V, d, dtype=torch.float64), torch.zeros(V, d, dtype=torch.float64)
        total.index_add_(0, i, x)
        size.index_add_(0, i, x.abs())
        n = torch.bincount(i, minlength=V)[:V].double()
        got = rows[w, seg].view(V, d).cpu()
        if accumulate:
            old = before[w, seg].view(V, d).cpu()
            assert torch.equal(got[n == 0], old[n == 0])
            total, size = total + old.double(), size + old.double().abs()
        else:
            assert bool((got[n == 0] == 0).all())
        assert bool(((got.double() - total).abs() <= (n + 3)[:, None] * 2.0 ** -24 * size).all())
    again = before.clone()
    ws.fill_(0xFF)
    nf.nf_embedding_grad(dy, ids, again, lead, V, ws, scale=scale, padding_id=padding, accumulate=accumulate)
    assert torch.equal(again, rows)


@pytest.mark.parametrize("dy_type", list(TYPES))
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("W,T,V,d,lead,extra", [
    (1, 1, 1, 1, 0, 0), (1, 1, 300, 64, 0, 0), (2, 63, 5, 33, 3, 0), (3, 64, 1000, 256, 4, 4), (2, 65, 64, 260, 8, 0),
    (1, 1024, 40, 128, 0, 0), (4, 1025, 257, 68, 0, 0), (1, 4096, 70_000, 16, 1, 3), (1, 4097, 3, 20, 0, 0),
    (5, 0, 11, 12, 4, 0), (1, 2000, 2000, 515, 517, 0)])
def test_grad(W, T, V, d, lead, extra, accumulate, dy_type):
    check_grad(W, T, V, d, dy_type, lead=lead, extra=extra, accumulate=accumulate, seed=T + d)


@pytest.mark.parametrize("T", [16_384, 16_385, 50_000, 70_001])
def test_grad_many_tokens(T):
    """One sorted run, and two to five merged ones; ids skewed so that stretches pass many chunks."""
    u = torch.rand(2, T, generator=torch.Generator().manual_seed(T))
    ids = (5000.0 ** u - 1).long() * 7 % 5000
    check_grad(2, T, 5000, 24, "bf16", ids=ids, seed=3)


@pytest.mark.parametrize("T", [64, 127, 128, 129, 1000, 20_000])
def test_grad_one_id(T):
    """Every token of one id: whole chunks, and edges of every length before and after them."""
    for first in (0, 1, 15, 16, 63, 64):
        ids = torch.full((1, T), 6)
        ids[0, :min(first, T - 1)] = 2
        check_grad(1, T, 9, 260, "f16", ids=ids, seed=first)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("d", [255, 257, 511, 513, 1023, 16_385, 25_345, 50_945])
def test_grad_wide_rows(d, accumulate):
    """Rows of many blocks' columns, of which the last may have a single one more than whole blocks do."""
    check_grad(2, 300, 3, d, lead=1, accumulate=accumulate, seed=d)


@pytest.mark.parametrize("kind", [torch.int32, torch.int64])
def test_grad_padding_and_outside(kind):
    g = torch.Generator().manual_seed(2)
    ids = torch.randint(-4, 24, (3, 700), generator=g)
    check_grad(3, 700, 20, 36, ids=ids, kind=kind, padding=7)
    check_grad(3, 700, 20, 36, ids=torch.full((3, 700), -1), kind=kind)            # no token at all
    check_grad(3, 700, 20, 36, ids=torch.full((3, 700), 20), kind=kind, accumulate=True)
    check_grad(3, 700, 20, 36, ids=torch.full((3, 700), 7), kind=kind, padding=7)  # all of them padding
    if kind == torch.int64:
        far = ids + (torch.arange(700) % 3 == 0) * 2 ** 32
        check_grad(3, 700, 20, 36, ids=far)


def test_grad_infinities_stay_in_their_rows():
    dy = torch.ones(1, 200, 8, device=DEV)
    dy[0, 17, 3], dy[0, 40, 2] = float("inf"), float("nan")
    ids = (torch.arange(200, device=DEV) % 10)[None]
    rows = torch.empty(1, 80, device=DEV)
    nf.nf_embedding_grad(dy, ids, rows, 0, 10, nf.empty_workspace(nf.nf_embedding_workspace_bytes(1, 200, 10, 8)))
    want = torch.full((10, 8), 20.0)
    want[7, 3], want[0, 2] = float("inf"), float("nan")
    assert torch.equal(rows.view(10, 8).cpu().nan_to_num(nan=-1.0), want.nan_to_num(nan=-1.0))


def test_grad_is_the_lookups():
    """L(table) = sum c * lookup(table) is linear: its difference along any direction is grad . direction."""
    g = torch.Generator().manual_seed(4)
    V, d, T = 40, 48, 300
    table, way = torch.randn(V, d, generator=g).to(DEV), torch.randn(V, d, generator=g).to(DEV)
    c = torch.randn(T, d, generator=g).to(DEV)
    ids = torch.randint(-1, V, (T,), generator=g).to(DEV)
    up, down = torch.empty(T, d, device=DEV), torch.empty(T, d, device=DEV)
    h = 0.5
    nf.nf_embedding_lookup(table + h * way, ids, up, scale=3.0)
    nf.nf_embedding_lookup(table - h * way, ids, down, scale=3.0)
    rows = torch.empty(1, V * d, device=DEV)
    ws = nf.empty_workspace(nf.nf_embedding_workspace_bytes(1, T, V, d))
    nf.nf_embedding_grad(c[None], ids[None], rows, 0, V, ws, scale=3.0)
    by_difference = float((c.double() * (up.double() - down.double())).sum() / (2 * h))
    by_gradient = float((rows.view(V, d).double() * way.double()).sum())
    # every product and sum rounded once: 2^-24 of their absolute values, some tokens a row
    size = float((c.abs().double() * (up.abs() + down.abs()).double()).sum() / (2 * h))
    assert abs(by_difference - by_gradient) <= 40 * 2.0 ** -24 * size


def test_graph_replays():
    W, T, V, d = 2, 500, 60, 32
    dy, ids = torch.randn(W, T, d, device=DEV), torch.randint(0, V, (W, T), device=DEV)
    rows, want = torch.empty(W, V * d, device=DEV), torch.empty(W, V * d, device=DEV)
    ws = nf.empty_workspace(nf.nf_embedding_workspace_bytes(W, T, V, d))
    nf.nf_embedding_grad(dy, ids, rows, 0, V, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nf.nf_embedding_grad(dy, ids, rows, 0, V, ws)
    for k in range(4):
        dy.copy_(torch.randn(W, T, d))
        ids.copy_(torch.randint(0, V // (k + 1), (W, T)))
        nf.nf_embedding_grad(dy, ids, want, 0, V, ws)
        rows.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(rows, want)


@pytest.mark.parametrize("accumulate", [False, True])
def test_segment_past_32_bits(accumulate):
    """A table of more than 2^31 elements, at an odd place in the row: the last ids' rows."""
    V, d, lead = 1_100_000, 2048, 5
    rows = torch.full((1, lead + V * d + 3), 2.0, device=DEV)
    ids = torch.tensor([[V - 1, 3, V - 1, 1_048_576]], device=DEV)
    dy = torch.arange(4, device=DEV).float()[None, :, None].expand(1, 4, d).contiguous()
    ws = nf.empty_workspace(nf.nf_embedding_workspace_bytes(1, 4, V, d))
    nf.nf_embedding_grad(dy, ids, rows, lead, V, ws, accumulate=accumulate)
    base = 2.0 if accumulate else 0.0
    seg = rows[0, lead:lead + V * d].view(V, d)
    assert bool((seg[V - 1] == 2 + base).all()) and bool((seg[3] == 1 + base).all())
    assert bool((seg[1_048_576] == 3 + base).all()) and bool((seg[1_048_575] == base).all())
    assert bool((seg[V - 2] == base).all()) and bool((rows[0, lead + V * d:] == 2.0).all())
    assert bool((rows[0, :lead] == 2.0).all())


def test_grad_one_token_each():
    """A dimension of one element has any stride: [W, 1] as the transpose of [1, W]."""
    W, V, d = 3, 7, 20
    ids = torch.tensor([[4, 0, 4]], device=DEV).t()
    assert ids.stride(-1) != 1
    dy = torch.randn(W, 1, d, device=DEV)
    rows = torch.full((W, V * d), float("nan"), device=DEV)
    nf.nf_embedding_grad(dy, ids, rows, 0, V, nf.empty_workspace(nf.nf_embedding_workspace_bytes(W, 1, V, d)))
    want = torch.zeros(W, V, d, device=DEV)
    for w, i in enumerate((4, 0, 4)):
        want[w, i] = dy[w, 0]
    assert torch.equal(rows.view(W, V, d), want)
