"""The example's training steps, every stage of them against a plain one from what the trainer itself held before it.

A falling loss does not show that each part works: the head alone brings it down.  Here the workers' rows are compared
with torch's gradients of a lookup by indexing and a table gradient summed in 64 bits, the reduced row with the oracle,
momentum and parameters with the definition of their step in 64 bits; and each stage has to have changed something.

Tolerances, relative in the 2-norm.  Rows: the same torch operations from an equal lookup, 1e-4 in case one of them adds
in another order (FP32 sums of at most 1,000 terms: 1,000 x 2^-24).  Momentum: two roundings.  Matrices: 3e-3 of the
orthogonalised update (11-bit operands).  Table and head: three roundings of numbers of the parameters' size.
"""
import importlib.util
import os

import numpy as np
import pytest
import torch

import oracle as nfo
import paper_2606_25759_amd as nf
from tests.test_gpu_orthogonal_tiles import COEF, definition, off

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ULP = 2.0 ** -24


def example():
    spec = importlib.util.spec_from_file_location("train_small", os.path.join(ROOT, "examples", "train_small.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain_rows(t, theta, ids, targets):
    """Every worker's gradient, by name."""
    rows = []
    for w in range(t.W):
        p = {k: t.view(theta, k).clone().requires_grad_(True) for k in ("up", "down", "head")}
        x = (t.view(theta, "table")[ids[w]] * t.scale).requires_grad_(True)
        y = x + torch.relu(x @ p["up"].t()) @ p["down"].t()
        loss = torch.nn.functional.cross_entropy(y @ p["head"].t(), targets[w])
        dx, *g = torch.autograd.grad(loss, [x, *p.values()])
        table = torch.zeros(t.V, t.d, dtype=torch.float64, device=theta.device)
        table.index_add_(0, ids[w], dx.double() * t.scale)
        rows.append({"table": table, **dict(zip(p, g))})
    return rows


def oracle_out(t, format):
    g, mask = t.rows.cpu().numpy(), t.mask.cpu().numpy().view(np.uint64)
    pol = nfo.policy(fp32_op=nf.NF_FP32_MEAN, format=format)
    reduce = nfo.reduce_bucket_ternary if format == nf.NF_FORMAT_TERNARY else nfo.reduce_bucket
    parts = []
    for at in range(0, t.n, t.bucket_n):
        end = min(at + t.bucket_n, t.n)
        parts.append(reduce(np.ascontiguousarray(g[:, at:end]), mask[at // 64:(end + 63) // 64], pol)["out"])
    return np.concatenate(parts)


@pytest.mark.parametrize("format", [nf.NF_FORMAT_BINARY, nf.NF_FORMAT_TERNARY])
def test_steps(format):
    t = example().Trainer(format=format, seed=3)
    for _ in range(4):
        theta, momentum, state = t.theta.clone(), t.momentum.clone(), t.gen.get_state()
        t.rows.fill_(float("nan"))
        t.rows[:, t.n:] = 0.0
        loss = t.step()
        after = t.gen.get_state()
        t.gen.set_state(state)
        ids, targets = t.batch()
        t.gen.set_state(after)
        assert loss == loss

        for w, want in enumerate(plain_rows(t, theta, ids, targets)):
            for name, g in want.items():
                assert float(torch.linalg.vector_norm(g)) > 0
                assert off(t.view(t.rows[w], name), g.double()) <= 1e-4, (w, name)

        ref = oracle_out(t, format)
        out = t.out.cpu().numpy()
        assert np.allclose(out, ref, rtol=1e-6, atol=0) and np.count_nonzero(out) > t.n // 2

        for name in ("table", "up", "down", "head"):
            g, before = t.view(t.out, name).double(), t.view(theta, name).double()
            m = float(np.float32(0.9)) * t.view(momentum, name).double() + g
            assert off(t.view(t.momentum, name), m) <= 2 * ULP, name
            if name in ("up", "down"):
                step = t.lr * 0.2 * max(g.shape) ** 0.5 * definition(g + 0.9 * m, [COEF] * 5)
                slack = 3e-3
            else:
                step, slack = 20 * t.lr * m, 0.0
            far = torch.linalg.vector_norm(t.view(t.theta, name).double() - (before - step))
            size, moved = torch.linalg.vector_norm(before), torch.linalg.vector_norm(step)
            allowed = float(slack * moved + 3 * ULP * (size + moved))
            assert float(moved) > 50 * allowed, name  # a step left out, or half of one, would show
            assert float(far) <= allowed, (name, float(far), allowed)
