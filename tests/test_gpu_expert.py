"""nf_expert_product and nf_expert_grad against plain products in 64 bits.

An FP32 sum of L products is off by at most (L + 2) 2^-23 times the sum of
the products' absolute values, in whatever order it is taken (2^-23: an
addition on the matrix cores need not round to nearest; 2 for the product's
own rounding and what is accumulated onto), and its rounding to the result's
type by half a step of it.
"""
import pytest
import torch

import paper_2606_25759_amd as nf

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def offsets_of(sizes, kind=torch.int32, start=0):
    """[W][E] sizes -> [W, E + 1] offsets."""
    s = torch.tensor(sizes, dtype=torch.int64)
    zero = torch.full((s.shape[0], 1), start, dtype=torch.int64)
    return torch.cat([zero, start + s.cumsum(1)], 1).to(kind).to(DEV)


def random_sizes(g, W, E, T):
    sizes = []
    for _ in range(W):
        cut = torch.sort(torch.randint(0, T + 1, (E + 1,), generator=g)).values
        sizes.append([int(b - a) for a, b in zip(cut[:-1], cut[1:])])
    return sizes


def strided(g, shape, kind, extra, scale=1.0):
    """A tensor whose rows are `extra` elements apart from being contiguous, and the buffer around it."""
    big = (torch.randn(*shape[:-1], shape[-1] + extra, generator=g) * scale).to(kind).to(DEV)
    return big[..., :shape[-1]], big


def close(got, want, size, length):
    eps = torch.finfo(got.dtype).eps / 2
    tiny = torch.finfo(got.dtype).smallest_normal * eps  # below it the steps stay the same
    allowed = (length + 2) * 2.0 ** -23 * size
    allowed = allowed + eps * (want.abs() + allowed) + tiny
    bad = ~((got.double() - want).abs() <= allowed)
    assert not bool(bad.any()), (int(bad.sum()), float((got.double() - want).abs().max()))


def check_product(W, E, T, n, k, back, kind="bf16", out="bf16", sizes=None, offsets=torch.int32, extra=0, start=0,
                  seed=0, stream=None):
    g = torch.Generator().manual_seed(seed)
    sizes = random_sizes(g, W, E, T) if sizes is None else sizes
    off = offsets_of(sizes, offsets, start)
    x, _ = strided(g, (W, T, n if back else k), TYPES[kind], extra)
    w, _ = strided(g, (E, n, k), TYPES[kind], extra)
    y, around = strided(g, (W, T, k if back else n), TYPES[out], extra)
    before = around.clone()
    nf.nf_expert_product(x, w, off, y, transposed=back, stream=stream)
    torch.cuda.synchronize()
    want, size = before[..., :y.shape[-1]].double(), torch.zeros(y.shape, dtype=torch.float64, device=DEV)
    touched = torch.zeros(W, T, dtype=torch.bool)
    for i in range(W):
        at = start
        for e, c in enumerate(sizes[i]):
            m = w[e].double() if back else w[e].double().t().contiguous()
            rows = x[i, at:at + c].double()
            want[i, at:at + c] = rows @ m
            size[i, at:at + c] = rows.abs() @ m.abs()
            touched[i, at:at + c] = True
            at += c
    touched = touched.to(DEV)
    close(y, want, size, n if back else k)
    assert torch.equal(y[~touched], before[..., :y.shape[-1]][~touched])  # no expert's rows
    assert torch.equal(around[..., y.shape[-1]:], before[..., y.shape[-1]:])
    return y


PRODUCTS = [  # W, E, T, n, k, extra
    (1, 1, 1, 1, 1, 0), (1, 3, 1, 16, 16, 0), (1, 8, 16, 64, 32, 0), (2, 5, 40, 33, 17, 0), (1, 4, 130, 128, 64, 0),
    (1, 4, 300, 136, 72, 8), (3, 7, 257, 100, 131, 3), (1, 2, 1000, 260, 520, 0), (1, 66, 200, 40, 24, 0),
    (1, 130, 97, 8, 200, 0), (1, 3, 700, 512, 256, 0), (1, 1, 513, 257, 255, 1), (2, 2, 0, 16, 16, 0)]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f32"), ("f32", "f16"),
                                      ("bf16", "f16")])
@pytest.mark.parametrize("W,E,T,n,k,extra", PRODUCTS)
def test_product(W, E, T, n, k, extra, kind, out, back):
    check_product(W, E, T, n, k, back, kind, out, extra=extra, seed=T + n,
                  offsets=torch.int64 if T % 2 else torch.int32)


WIDE_PRODUCTS = [  # W, E, T, n, k, back
    (1, 4, 16_500, 1032, 264, False), (1, 4, 16_500, 264, 1032, True), (2, 3, 9_000, 1024, 200, False),
    (2, 3, 9_000, 72, 1024, True), (1, 2, 66_000, 192, 64, False), (1, 30, 8_000, 2056, 320, False)]


@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("W,E,T,n,k,back", WIDE_PRODUCTS)
def test_product_wide_tiles(W, E, T, n, k, back, kind, out):
    """Sizes that take tiles of 256, their lengths ending inside stages and tiles; an expert of a single row."""
    g = torch.Generator().manual_seed(T)
    sizes = random_sizes(g, W, E, T - 300)
    sizes[0][0] = 1 if E > 2 else 40_000 if T > 60_000 else sizes[0][0]
    assert all(sum(row) <= T for row in sizes)
    check_product(W, E, T, n, k, back, kind, out, sizes=sizes, seed=1)


F32_PRODUCTS = [  # W, E, T, n, k, back
    (8, 3, 1024, 1664, 48, False), (8, 3, 1024, 44, 1660, True), (8, 3, 1024, 1601, 35, False), (8, 3, 1025, 37, 1603, True)]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("W,E,T,n,k,back", F32_PRODUCTS)
def test_product_f32_large_tiles(W, E, T, n, k, back, out):
    """FP32 in tiles of 128, straight into LDS and by registers; uneven experts, rows of none before and behind them."""
    check_product(W, E, T, n, k, back, "f32", out, seed=n)
    check_product(W, E, T, n, k, back, "f32", out, sizes=[[1, 0, T - 130], [0, T, 0]] * (W // 2), start=0, seed=k)


OTHER_PRODUCTS = [  # W, E, T, n, k, extra
    (1, 1, 1, 512, 2048, 0), (1, 2, 70, 320, 1030, 2), (1, 6, 1500, 520, 264, 0), (2, 5, 900, 515, 260, 1),
    (1, 3, 3000, 768, 1032, 0), (1, 2, 3000, 769, 515, 3), (1, 3, 4000, 512, 520, 0), (1, 3, 4000, 513, 515, 0)]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("W,E,T,n,k,extra", OTHER_PRODUCTS)
def test_product_other_tiles(W, E, T, n, k, extra, kind, back):
    """Sizes that take tiles of 32, of 128 x 32 and of 128, straight into LDS and by registers."""
    check_product(W, E, T, n, k, back, kind, "f32", extra=extra, seed=n + k)


@pytest.mark.parametrize("back", [False, True])
def test_sizes_at_the_edges_of_tiles(back):
    for sizes in ([0, 0, 0, 0], [31, 32, 33, 1], [127, 0, 128, 129], [255, 256, 257, 0], [0, 0, 513, 0], [1, 1, 1, 1]):
        T = sum(sizes) + 5
        check_product(1, 4, T, 72, 88, back, sizes=[sizes], start=0)
        check_product(1, 4, T, 72, 88, back, sizes=[sizes], start=5)  # rows before the first expert's, none behind


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kind", list(TYPES))
def test_no_reduction_gives_zeros(back, kind):
    n, k = (0, 24) if back else (24, 0)
    y = check_product(1, 3, 50, n, k, back, kind, "f32", sizes=[[20, 0, 25]])
    assert bool((y[0, :45] == 0).all())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("back", [False, True])
def test_infinities_and_nan_stay_in_their_rows(kind, back):
    """A row with a NaN beside finite ones, in lengths that end inside a stage: what lies past an end is not read."""
    for n, k in ((96, 136), (40, 50), (200, 72)):
        rows, cols = (n, k) if back else (k, n)
        x = torch.ones(1, 60, rows + 16, dtype=TYPES[kind], device=DEV)
        x[..., rows:] = float("nan")  # behind each row's end
        x[0, 7, 3], x[0, 30, rows - 1] = float("nan"), float("inf")
        w = torch.ones(3, n, k + 8, dtype=TYPES[kind], device=DEV)
        w[..., k:] = float("nan")
        w[1] = 2.0
        w[1, :, k:] = float("nan")
        y = torch.zeros(1, 60, cols, device=DEV)
        off = torch.tensor([0, 20, 45, 60], device=DEV, dtype=torch.int32)
        nf.nf_expert_product(x[..., :rows], w[..., :k], off, y, transposed=back)
        want = torch.full((60, cols), float(rows), device=DEV)
        want[20:45] *= 2
        want[7], want[30] = float("nan"), float("inf")
        assert torch.equal(torch.nan_to_num(y[0], nan=-5.0), torch.nan_to_num(want, nan=-5.0))


@pytest.mark.parametrize("kind", list(TYPES))
def test_smallest_and_largest_elements(kind):
    """Subnormal elements count, and sums of the largest FP16 ones do not overflow on the way."""
    t = TYPES[kind]
    small, large = torch.finfo(t).tiny / 4, 2.0 ** 100 if kind != "f16" else 2.0 ** 15
    for T, n, k in ((3, 32, 64), (300, 256, 128), (70, 33, 17)):
        x = torch.full((T, k), small, dtype=t, device=DEV)
        w = torch.full((1, n, k), large, dtype=t, device=DEV)
        off = torch.tensor([0, T], dtype=torch.int32, device=DEV)
        y = torch.empty(T, n, device=DEV)
        nf.nf_expert_product(x, w, off, y)
        assert torch.equal(y, torch.full_like(y, k * small * large))
        dx = torch.empty(T, k, device=DEV)
        nf.nf_expert_product(torch.full((T, n), small, dtype=t, device=DEV), w, off, dx, transposed=True)
        assert torch.equal(dx, torch.full_like(dx, n * small * large))
        rows = torch.empty(1, n * k, device=DEV)
        nf.nf_expert_grad(torch.full((T, n), large, dtype=t, device=DEV), x, off, rows, 0,
                          nf.empty_workspace(nf.nf_expert_grad_workspace_bytes(1, T, 1, n, k)))
        assert torch.equal(rows, torch.full_like(rows, T * small * large))
    x = torch.full((4, 64), 60_000.0, dtype=t, device=DEV)
    y = torch.empty(4, 32, device=DEV)
    w = torch.full((1, 32, 64), 60_000.0, dtype=t, device=DEV)
    nf.nf_expert_product(x, w, torch.tensor([0, 4], dtype=torch.int32, device=DEV), y)
    want = 64 * float(x[0, 0]) * float(w[0, 0, 0])
    assert bool(((y.double() - want).abs() <= 66 * 2.0 ** -23 * want).all())


def check_grad(W, E, T, n, k, kind="bf16", sizes=None, offsets=torch.int32, extra=0, lead=0, gap=0, accumulate=False,
               start=0, seed=0):
    g = torch.Generator().manual_seed(seed)
    sizes = random_sizes(g, W, E, T) if sizes is None else sizes
    off = offsets_of(sizes, offsets, start)
    dy, _ = strided(g, (W, T, n), TYPES[kind], extra)
    x, _ = strided(g, (W, T, k), TYPES[kind], extra)
    each = n * k + gap
    rows = torch.randn(W, (lead + E * each + 11) // 4 * 4, generator=g).to(DEV)
    before = rows.clone()
    ws = nf.empty_workspace(nf.nf_expert_grad_workspace_bytes(W, T, E, n, k))
    ws.fill_(0xFF)
    nf.nf_expert_grad(dy, x, off, rows, lead, ws, accumulate=accumulate, matrix_stride=each)
    outside = torch.ones(rows.shape[1], dtype=torch.bool)
    for e in range(E):
        outside[lead + e * each:lead + e * each + n * k] = False
    assert torch.equal(rows[:, outside.to(DEV)], before[:, outside.to(DEV)])
    for i in range(W):
        at = start
        for e, c in enumerate(sizes[i]):
            a, b = dy[i, at:at + c].double(), x[i, at:at + c].double()
            want, size = a.t() @ b, a.abs().t() @ b.abs()
            seg = slice(lead + e * each, lead + e * each + n * k)
            got = rows[i, seg].view(n, k)
            if accumulate and c == 0:
                assert torch.equal(got.view(torch.int32), before[i, seg].view(n, k).view(torch.int32))
            if accumulate:
                old = before[i, seg].view(n, k).double()
                want, size = want + old, size + old.abs()
            elif c == 0:
                assert bool((got == 0).all())
            close(got, want, size, c)
            at += c
    again = before.clone()
    ws.fill_(0x7F)
    nf.nf_expert_grad(dy, x, off, again, lead, ws, accumulate=accumulate, matrix_stride=each)
    assert torch.equal(again, rows)


GRADS = [  # W, E, T, n, k, extra, lead, gap
    (1, 1, 1, 1, 1, 0, 0, 0), (1, 3, 40, 16, 16, 0, 0, 0), (2, 5, 100, 33, 17, 0, 3, 0), (1, 4, 700, 136, 72, 8, 4, 8),
    (3, 7, 257, 100, 131, 3, 517, 5), (1, 2, 3000, 130, 260, 0, 0, 0), (1, 66, 200, 40, 24, 0, 1, 0),
    (1, 2, 4100, 64, 64, 0, 0, 0), (1, 3, 700, 512, 256, 0, 0, 0), (2, 2, 0, 16, 16, 0, 2, 0)]


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("W,E,T,n,k,extra,lead,gap", GRADS)
def test_grad(W, E, T, n, k, extra, lead, gap, kind, accumulate):
    check_grad(W, E, T, n, k, kind, extra=extra, lead=lead, gap=gap, accumulate=accumulate, seed=T + n,
               offsets=torch.int64 if T % 2 else torch.int32)


WIDE_GRADS = [(1, 4, 900, 2056, 2040), (2, 33, 300, 1032, 1048), (1, 64, 500, 512, 520)]  # W, E, T, n, k
SHARED_GRADS = [(1, 2, 9000, 72, 40), (2, 1, 5000, 130, 70), (1, 3, 12_000, 129, 71)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("W,E,T,n,k", SHARED_GRADS)
def test_grad_shared_tokens(W, E, T, n, k, kind):
    check_grad(W, E, T, n, k, kind, lead=5, seed=T)
    check_grad(W, E, T, n, k, kind, accumulate=True, seed=T)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("W,E,T,n,k", WIDE_GRADS)
def test_grad_wide_tiles(W, E, T, n, k, kind, accumulate):
    """Sizes that take tiles of 256: experts by length over all XCDs, and (few tiles an expert) one after the other."""
    check_grad(W, E, T, n, k, kind, lead=3, accumulate=accumulate, seed=E)


@pytest.mark.parametrize("kind", list(TYPES))
def test_grad_shares_of_uneven_experts(kind):
    """Tokens shared between blocks: experts of no share, of one, of several and of all."""
    for sizes in ([0, 15_000, 0, 3], [256, 257, 4512, 513], [0, 0, 0, 6900], [1, 0, 1, 255]):
        check_grad(1, 4, 16_000, 40, 72, kind, sizes=[sizes])
        check_grad(1, 4, 16_000, 40, 72, kind, sizes=[sizes], start=9, accumulate=True, lead=1)


def test_grad_infinities_stay_in_their_expert():
    """A NaN in one expert's last token leaves the next expert's sums alone, and what lies behind rows is not read."""
    for kind in TYPES.values():
        dy = torch.full((1, 90, 40), float("nan"), dtype=kind, device=DEV)
        x = torch.full((1, 90, 56), float("nan"), dtype=kind, device=DEV)
        dy[0, :80, :32], x[0, :80, :48] = 1.0, 2.0
        x[0, 29, 5] = float("nan")
        off = torch.tensor([0, 30, 33, 80], dtype=torch.int32, device=DEV)
        rows = torch.zeros(1, 3 * 32 * 48, device=DEV)
        ws = nf.empty_workspace(nf.nf_expert_grad_workspace_bytes(1, 90, 3, 32, 48))
        nf.nf_expert_grad(dy[..., :32], x[..., :48], off, rows, 0, ws)
        got = rows.view(3, 32, 48)
        assert bool(got[0, :, 5].isnan().all()) and int(got.isnan().sum()) == 32
        got[0, :, 5] = 60.0
        assert torch.equal(got, torch.tensor([60.0, 6.0, 94.0], device=DEV)[:, None, None].expand(3, 32, 48))


def test_offsets_that_make_no_sense_touch_nothing_else():
    """Values outside [0, T] and descending ones: every access stays inside the tensors."""
    T, E, n, k = 70, 5, 24, 40
    x, w = torch.randn(1, T, k, device=DEV).bfloat16(), torch.randn(E, n, k, device=DEV).bfloat16()
    for values in ([-9, 20, 30, 10, 50, 900], [60, 50, 40, 30, 20, 10], [0, 70, 0, 70, 0, 70],
                   [2 ** 31 - 1, -2 ** 31, 5, 2 ** 31 - 1, 7, 70]):
        off = torch.tensor(values, device=DEV, dtype=torch.int32)
        y = torch.full((T + 20, n), 3.0, device=DEV)
        nf.nf_expert_product(x[0], w, off, y[10:-10])
        rows = torch.full((1, E * n * k + 16), 3.0, device=DEV)
        ws = nf.empty_workspace(nf.nf_expert_grad_workspace_bytes(1, T, E, n, k))
        nf.nf_expert_grad(x[..., :n].contiguous(), x, off, rows, 8, ws)
        assert bool((y[:10] == 3).all()) and bool((y[-10:] == 3).all())
        assert bool((rows[:, :8] == 3).all()) and bool((rows[:, -8:] == 3).all())
    for values in ([0, 9000, 0, 9000, 0, 9000], [9000, 0, 9000, -1, 10_000, 3]):  # with shared tokens, larger tiles
        T, n, k = 9000, 72, 40
        off = torch.tensor(values, device=DEV)
        need = nf.nf_expert_grad_workspace_bytes(1, T, E, n, k)
        assert need > 0
        ws = torch.full((need + 512,), 0x55, dtype=torch.uint8, device=DEV)
        x, dy = torch.randn(T, k, device=DEV).half(), torch.randn(T, n, device=DEV).half()
        rows = torch.full((1, E * n * k + 16), 3.0, device=DEV)
        nf.nf_expert_grad(dy, x, off, rows, 8, ws[256:256 + need])
        assert bool((rows[:, :8] == 3).all()) and bool((rows[:, -8:] == 3).all())
        assert bool((ws[:256] == 0x55).all()) and bool((ws[256 + need:] == 0x55).all())
        y = torch.full((T + 20, n), 3.0, device=DEV)
        nf.nf_expert_product(x, torch.randn(E, n, k, device=DEV).half(), off, y[10:-10])
        assert bool((y[:10] == 3).all()) and bool((y[-10:] == 3).all())


def test_gradients_against_differences():
    """The two gradients are those of the product: central differences of sum(c y) in FP64 of FP32 results."""
    W, E, T, n, k = 1, 3, 24, 20, 28
    g = torch.Generator().manual_seed(5)
    off = offsets_of([[9, 0, 13]])
    x, w = torch.randn(W, T, k, generator=g).to(DEV), torch.randn(E, n, k, generator=g).to(DEV)
    c = torch.randn(W, T, n, generator=g).to(DEV)
    c[:, 22:] = 0

    def value(x, w):
        y = torch.zeros(W, T, n, device=DEV)
        nf.nf_expert_product(x, w, off, y)
        return float((y.double() * c.double()).sum())

    dx = torch.zeros(W, T, k, device=DEV)
    nf.nf_expert_product(c, w, off, dx, transposed=True)
    rows = torch.zeros(W, E * n * k, device=DEV)
    nf.nf_expert_grad(c, x, off, rows, 0, nf.empty_workspace(nf.nf_expert_grad_workspace_bytes(W, T, E, n, k)))
    dw = rows.view(E, n, k)
    # the function is linear in each, so a step of 1/2 has no error of its own; 22 x 20 FP32 results are off by at
    # most 30 2^-23 28 max|x w| max|c| each, about 2e-3 in all
    for at in ((0, 3, 4), (0, 10, 27), (0, 21, 0)):
        d = torch.zeros_like(x)
        d[at] = 0.5
        assert abs(value(x + d, w) - value(x - d, w) - float(dx[at])) < 4e-3
    for at in ((0, 3, 4), (2, 19, 27), (1, 0, 0)):
        d = torch.zeros_like(w)
        d[at] = 0.5
        assert abs(value(x, w + d) - value(x, w - d) - float(dw[at])) < 4e-3
    assert bool((dw[1] == 0).all()) and bool((dx[0, 22:] == 0).all())


def test_other_stream_and_graph_replays():
    """Captured once, replayed with other inputs, sizes and eager work between: equal to eager calls."""
    W, E, T, n, k = 2, 4, 900, 96, 64
    side = torch.cuda.Stream()
    x, dy = (torch.empty(W, T, c, dtype=torch.bfloat16, device=DEV) for c in (k, n))
    w = torch.randn(E, n, k, device=DEV).bfloat16()
    off = torch.zeros(W, E + 1, dtype=torch.int32, device=DEV)
    y, dx = torch.zeros(W, T, n, device=DEV), torch.zeros(W, T, k, device=DEV)
    rows = torch.zeros(W, E * n * k, device=DEV)
    ws = nf.empty_workspace(nf.nf_expert_grad_workspace_bytes(W, T, E, n, k))

    def calls():
        nf.nf_expert_product(x, w, off, y)
        nf.nf_expert_product(dy, w, off, dx, transposed=True)
        nf.nf_expert_grad(dy, x, off, rows, 0, ws)

    def fill(seed):
        g = torch.Generator().manual_seed(seed)
        x.copy_(torch.randn(x.shape, generator=g))
        dy.copy_(torch.randn(dy.shape, generator=g))
        off.copy_(offsets_of(random_sizes(g, W, E, T)))
        for t in (y, dx, rows):
            t.fill_(7.0)

    fill(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in range(4):
        fill(seed)
        calls()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, dx, rows)]
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((y, dx, rows), want):
            assert torch.equal(a, b)


def test_far_rows_and_matrices():
    """Elements past 2^31 of x, w and the gradient's row."""
    T, E, n, k = 40, 2, 16, 32
    far = 2 ** 31 + 64
    big = torch.empty(far + 4096, dtype=torch.bfloat16, device=DEV)
    w = big.as_strided((E, n, k), (far, k, 1))
    w.copy_(torch.randn(E, n, k, device=DEV))
    x = torch.randn(1, T, k, device=DEV).bfloat16()
    off = torch.tensor([0, 15, 40], dtype=torch.int64, device=DEV)
    y = torch.empty(1, T, n, device=DEV)
    nf.nf_expert_product(x, w, off, y)
    size = torch.cat([x[0, :15].double().abs() @ w[0].double().abs().t(), x[0, 15:].double().abs() @ w[1].double().abs().t()])
    want = torch.cat([x[0, :15].double() @ w[0].double().t(), x[0, 15:].double() @ w[1].double().t()])
    close(y[0], want, size, k)
    step = far // (T - 1) // 64 * 64 + 64
    rows_apart = torch.empty((T - 1) * step + k, dtype=torch.bfloat16, device=DEV).as_strided((T, k), (step, 1))
    rows_apart.copy_(x[0])
    y2 = torch.empty(T, n, device=DEV)
    nf.nf_expert_product(rows_apart, w, off, y2)
    close(y2, want, size, k)
    del big, w, rows_apart
    rows = torch.full((1, far + n * k), 2.0, device=DEV)
    dy = torch.randn(1, T, n, device=DEV).bfloat16()
    nf.nf_expert_grad(dy, x, off, rows, 0, nf.empty_workspace(nf.nf_expert_grad_workspace_bytes(1, T, E, n, k)),
                      matrix_stride=far)
    a, b = dy[0, 15:].double(), x[0, 15:].double()
    close(rows[0, far:].view(n, k), a.t() @ b, a.abs().t() @ b.abs(), 25)
    assert bool((rows[0, n * k:n * k + 999] == 2).all())
