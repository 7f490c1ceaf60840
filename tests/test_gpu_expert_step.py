"""A training step of a layer of experts around the bucket reducer, every operator in its place:

    tokens gathered in the order of their experts -> two products with a ReLU between -> back -> the rows' gradients by
    the transposed products -> the matrices' gradients into the workers' rows -> each worker's row clipped in place by
    its own norm -> the reducer -> the matrices stepped by their orthogonalised gradient

Each stage is checked against its definition in 64 bits on what the stages before it gave, so that no error of one is
another's; then the whole step again, and from a captured graph, for equal bits.
"""
import numpy as np
import pytest
import torch

import paper_2606_25759_amd as nf
from tests.test_gpu_expert import close
from tests.test_gpu_norm import factor

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
W, T, E, D, H = 3, 500, 5, 96, 160
MAX_NORM = 0.05


class Step:
    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        rand = lambda s, *size: (torch.randn(*size, generator=g) * s).to(DEV)  # noqa: E731
        self.x, self.target = rand(1.0, W, T, D).bfloat16(), rand(1.0, W, T, D)
        self.choice = torch.randint(0, E - 1, (W, T), generator=g).to(DEV)  # the last expert is never chosen
        self.n = 2 * E * H * D
        self.up_at, self.down_at = 0, E * H * D
        self.theta = rand(0.1, self.n)
        self.momentum = torch.zeros(self.n, device=DEV)
        self.up, self.down = (torch.empty(E, *s, dtype=torch.bfloat16, device=DEV) for s in ((H, D), (D, H)))
        self.rows = torch.empty(W, self.n, device=DEV)
        self.hidden, self.dhidden = (torch.zeros(W, T, H, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        self.sorted, self.y, self.dx = (torch.zeros(W, T, D, dtype=torch.bfloat16, device=DEV) for _ in range(3))
        self.offsets = torch.zeros(W, E + 1, dtype=torch.int64, device=DEV)
        size = lambda *s: nf.nf_expert_grad_workspace_bytes(W, T, E, *s)  # noqa: E731
        self.ws = nf.empty_workspace(max(size(H, D), size(D, H)))
        self.plan = nf.norm_plan(list(self.rows), list(self.rows), range(W))
        self.norm_ws = nf.empty_workspace(nf.nf_grad_norm_workspace_bytes(self.plan))
        self.norms = torch.empty(W, device=DEV)
        self.bucket_n = self.n // 3 // 64 * 64
        nb = -(-self.n // self.bucket_n)
        # the FP32 route: what comes out is the rows' mean
        mask = nf.nf_mask_from_segments([0], [self.n], [0], self.n)
        self.mask = torch.from_numpy(mask.view(np.int64)).to(DEV)
        self.policy = nf.policy(fp32_op=nf.NF_FP32_MEAN)
        self.bits = torch.empty(W, (self.n + 63) // 64, dtype=torch.int64, device=DEV)
        self.out = torch.empty(self.n, device=DEV)
        self.stats = torch.empty(nb * W * nf.STATS_BYTES, dtype=torch.uint8, device=DEV)
        self.decisions = torch.empty(nb * nf.DECISION_BYTES, dtype=torch.uint8, device=DEV)
        self.reduce_ws = nf.empty_workspace(nf.nf_workspace_bytes_buckets(W, self.n, self.bucket_n))
        self.how = nf.orthogonal()
        self.matrix_ws = nf.empty_workspace(max(nf.nf_orthogonal_workspace_bytes(H, D, E, self.how),
                                                nf.nf_orthogonal_workspace_bytes(D, H, E, self.how)))

    def part(self, flat, name):
        return flat[:self.down_at].view(E, H, D) if name == "up" else flat[self.down_at:].view(E, D, H)

    def tokens(self):
        """Which rows each expert gets: the program's own work, between the library's calls."""
        self.order = torch.argsort(self.choice, dim=1, stable=True)
        ends = torch.stack([(self.choice <= e).sum(1) for e in range(E)], 1)
        self.offsets[:, 1:] = ends

    def run(self):
        self.up.copy_(self.part(self.theta, "up"))
        self.down.copy_(self.part(self.theta, "down"))
        for w in range(W):
            nf.nf_embedding_lookup(self.x[w], self.order[w], self.sorted[w])
        nf.nf_expert_product(self.sorted, self.up, self.offsets, self.hidden)
        self.hidden.relu_()
        nf.nf_expert_product(self.hidden, self.down, self.offsets, self.y)
        want = self.target.gather(1, self.order[..., None].expand(-1, -1, D))
        self.dy = ((self.y.float() - want) / (T * D)).bfloat16()
        nf.nf_expert_grad(self.dy, self.hidden, self.offsets, self.rows, self.down_at, self.ws)
        nf.nf_expert_product(self.dy, self.down, self.offsets, self.dhidden, transposed=True)
        self.dhidden.mul_(self.hidden > 0)
        nf.nf_expert_grad(self.dhidden, self.sorted, self.offsets, self.rows, self.up_at, self.ws)
        nf.nf_expert_product(self.dhidden, self.up, self.offsets, self.dx, transposed=True)
        self.before_clip = self.rows.clone()
        nf.nf_grad_norm_clip(self.plan, MAX_NORM, self.norms, self.norm_ws)
        nf.nf_route_buckets(self.rows, self.n, self.bucket_n, self.mask, self.policy, self.bits, None, self.out,
                            self.stats, self.decisions, self.reduce_ws)
        self.before_step = self.theta.clone()
        for name, shape in (("up", (H, D)), ("down", (D, H))):
            nf.nf_orthogonal_update(self.part(self.out, name), self.part(self.momentum, name),
                                    self.part(self.theta, name), nf.matrix_step(lr=0.02, scale=0.2 * max(shape) ** 0.5),
                                    self.how, self.matrix_ws)

    def results(self):
        return [t.clone() for t in (self.y, self.dx, self.dhidden, self.before_clip, self.norms, self.rows, self.out,
                                    self.momentum, self.theta)]


def groups(s):
    off = s.offsets.cpu().tolist()
    return [(w, e, slice(off[w][e], off[w][e + 1])) for w in range(W) for e in range(E)]


def test_step_stage_by_stage():
    s = Step(0)
    s.tokens()
    s.run()
    torch.cuda.synchronize()
    for w in range(W):
        assert torch.equal(s.sorted[w], s.x[w][s.order[w]])
        chosen = s.choice[w][s.order[w]]
        assert all(bool((chosen[at] == e).all()) for v, e, at in groups(s) if v == w)
    for name, x, m, y, length in (("down", s.hidden, s.down, s.y, H), ("dx", s.dhidden, s.up.transpose(1, 2), s.dx, H)):
        for w, e, at in groups(s):
            a, b = x[w, at].double(), m[e].double().t().contiguous()
            close(y[w, at], a @ b, a.abs() @ b.abs(), length)
    for w, e, at in groups(s):  # with the ReLU
        a, b = s.sorted[w, at].double(), s.up[e].double().t().contiguous()
        close(s.hidden[w, at], (a @ b).relu(), a.abs() @ b.abs(), D)
        a, b = s.dy[w, at].double(), s.down[e].double()
        on = (s.hidden[w, at] > 0).double()
        close(s.dhidden[w, at], (a @ b) * on, (a.abs() @ b.abs()) * on, D)
        for name, dy, x in (("up", s.dhidden, s.sorted), ("down", s.dy, s.hidden)):
            a, b = dy[w, at].double(), x[w, at].double()
            close(s.part(s.before_clip[w], name)[e], a.t() @ b, a.abs().t() @ b.abs(), at.stop - at.start)
    for w in range(W):
        norm = float(s.before_clip[w].double().square().sum().sqrt())
        assert abs(float(s.norms[w]) - norm) <= 1.001 * 2.0 ** -24 * norm and norm > MAX_NORM
        by = torch.tensor(factor(float(s.norms[w]), MAX_NORM), device=DEV)
        assert torch.equal(s.rows[w], s.before_clip[w] * by)
    assert bool((nf.decisions_host(s.decisions, -(-s.n // s.bucket_n))["route"] != nf.NF_ROUTE_LOWBIT).all())
    mean = s.rows.double().mean(0)  # an FP32 sum of W terms in some order, times 1 / W: four roundings
    assert bool(((s.out.double() - mean).abs() <= 4 * 2.0 ** -24 * s.rows.double().abs().mean(0) + 2.0 ** -149).all())
    for name, shape in (("up", (H, D)), ("down", (D, H))):
        for e in range(E):
            g = s.part(s.out, name)[e].double()
            u = g + 0.95 * g  # the first step's momentum is the gradient
            x = u / (u.norm() + 1e-7)
            a, b, c = 3.4445, -4.7750, 2.0315
            for _ in range(5):
                gram = x @ x.t()
                x = a * x + (b * gram + c * gram @ gram) @ x
            old = s.part(s.before_step, name)[e].double()
            moved = (s.part(s.theta, name)[e].double() - old) / (-0.02 * 0.2 * max(shape) ** 0.5)
            if e == E - 1:  # no token: no gradient, no step
                assert bool((moved == 0).all())
            else:
                # 2e-3 of its norm as nf_orthogonalize says, and the weights' FP32 rounding seen through lr scale
                assert float((moved - x).norm()) <= 2e-3 * float(x.norm()) + 2.0 ** -24 * float(old.norm()) / 0.05


def test_step_gradients_are_those_of_the_loss():
    """The chain of the three kinds of products against autograd in 64 bits: BF16 activations round four times on the
    way (2^-9 each), in a chain whose terms largely cancel: within 3% of a gradient's norm."""
    s = Step(1)
    s.tokens()
    s.run()
    for w in range(W):
        x = s.x[w].double().requires_grad_(True)
        up, down = (t.double().requires_grad_(True) for t in (s.up, s.down))
        loss = 0.0
        for e in range(E):
            at = s.choice[w] == e
            y = torch.relu(x[at] @ up[e].t()) @ down[e].t()
            loss = loss + 0.5 * (y - s.target[w][at].double()).square().sum() / (T * D)
        dx, dup, ddown = torch.autograd.grad(loss, [x, up, down])
        for got, want in ((s.dx[w], dx[s.order[w]]), (s.part(s.before_clip[w], "up"), dup),
                          (s.part(s.before_clip[w], "down"), ddown)):
            assert float((got.double() - want).norm()) <= 0.03 * float(want.norm())


def test_step_twice_and_captured():
    """The same bits from a second state, and from a graph that is replayed with eager steps of the other between."""
    a, b = Step(2), Step(2)
    for s in (a, b):
        s.tokens()
    a.run()
    first = a.results()
    b.run()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, b.results()))
    start = Step(2)
    b.theta.copy_(start.theta)
    b.momentum.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.run()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run()
    b.theta.copy_(start.theta)
    b.momentum.zero_()
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        if k:
            a.run()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a.results(), b.results())), k
