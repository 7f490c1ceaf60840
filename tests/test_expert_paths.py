"""Which kernels the expert products run: every one of them is reached by the sizes of the GPU tests, and the query
refuses what the calls do (no GPU needed)."""
import ctypes

import pytest

import paper_2606_25759_amd as nf
from tests import test_gpu_expert as t

CODES = {"f32": nf.NF_TYPE_F32, "bf16": nf.NF_TYPE_BF16, "f16": nf.NF_TYPE_F16}
OPS = (nf.NF_EXPERT_PRODUCT, nf.NF_EXPERT_TRANSPOSED)


def whole(kind, *lengths):
    return all(c % (4 if kind == "f32" else 8) == 0 for c in lengths)


def reached():
    found = set()

    def add(op, kind, W, T, E, n, k, lengths):
        i = nf.nf_expert_path(op, CODES[kind], W, T, E, n, k, whole(kind, *lengths))
        found.add((op, kind, i.tile_columns, i.tile_rows, i.direct, i.share > 0))

    for kind in CODES:
        for W, E, T, n, k, extra in t.PRODUCTS + t.OTHER_PRODUCTS:
            add(OPS[0], kind, W, T, E, n, k, (k, k + extra))
            add(OPS[1], kind, W, T, E, n, k, (n, k, n + extra, k + extra))
        for W, E, T, n, k, extra, _, _ in t.GRADS:
            add(nf.NF_EXPERT_GRAD, kind, W, T, E, n, k, (n, k, n + extra, k + extra))
        for W, E, T, n, k in t.SHARED_GRADS + (t.WIDE_GRADS if kind != "f32" else []):
            add(nf.NF_EXPERT_GRAD, kind, W, T, E, n, k, (n, k))
        for W, E, T, n, k, back in t.WIDE_PRODUCTS if kind != "f32" else []:
            add(OPS[back], kind, W, T, E, n, k, (n, k) if back else (k,))
        for W, E, T, n, k, back in t.F32_PRODUCTS if kind == "f32" else []:
            add(OPS[back], kind, W, T, E, n, k, (n, k) if back else (k,))
    return {f for f in found if f[2]}


def test_every_kernel_is_tested():
    want = set()
    for kind in CODES:
        for direct in (0, 1):
            for op in OPS:
                want |= {(op, kind, c, r, direct, False) for c, r in ((32, 32), (128, 32), (128, 128))}
            want |= {(nf.NF_EXPERT_GRAD, kind, 128, 128, direct, shared) for shared in (False, True)}
        if kind != "f32":
            want |= {(op, kind, 256, 256, 1, False) for op in (*OPS, nf.NF_EXPERT_GRAD)}
    got = reached()
    assert got == want, (sorted(want - got), sorted(got - want))


def test_shares_need_their_workspace():
    for W, E, T, n, k in t.SHARED_GRADS:
        i = nf.nf_expert_path(nf.NF_EXPERT_GRAD, nf.NF_TYPE_BF16, W, T, E, n, k)
        assert i.share >= 64 and nf.nf_expert_grad_workspace_bytes(W, T, E, n, k) > 0
    assert nf.nf_expert_grad_workspace_bytes(1, 100, 2, 64, 64) == 0


def test_refusals():
    good = [0, 1, 1, 10, 2, 8, 8, 1]
    for at, value in ((0, 3), (0, -1), (1, 3), (2, 0), (2, 256), (3, -1), (4, 4097), (5, -1), (6, 1 << 21), (7, 2)):
        args = list(good)
        args[at] = value
        info = nf.nf_expert_path_info()
        assert nf.load().nf_expert_path(*args, ctypes.byref(info)) == nf.NF_ERR_INVALID_ARG
    assert nf.load().nf_expert_path(*good, None) == nf.NF_ERR_INVALID_ARG
    with pytest.raises(nf.NFError) as e:
        nf.nf_expert_path(0, 1, 200, 1 << 24, 4, 2000, 64)
    assert e.value.status == nf.NF_ERR_UNSUPPORTED
    for args in ((0, 1, 1, 0, 2, 8, 8), (0, 1, 1, 5, 0, 8, 8), (0, 1, 1, 5, 2, 0, 8), (1, 1, 1, 5, 2, 8, 0), (2, 1, 1, 5, 2, 0, 8)):
        i = nf.nf_expert_path(*args)
        assert (i.tile_columns, i.tile_rows, i.direct, i.share) == (0, 0, 0, 0)
