"""Refusals of the embedding and orthogonalisation entry points: an error code
before anything is launched (no GPU needed), and the binding's own checks."""
import ctypes

import pytest
import torch

import paper_2606_25759_amd as nf

P = ctypes.c_void_p
F = ctypes.c_float
FAKE, ODD, WS = P(0x1000), P(0x1001), P(0x100000)  # never dereferenced: validation fails first
BIG = 1 << 40
INVALID, ALIGN, UNSUPPORTED, WORKSPACE = (nf.NF_ERR_INVALID_ARG, nf.NF_ERR_ALIGNMENT, nf.NF_ERR_UNSUPPORTED,
                                          nf.NF_ERR_WORKSPACE)


def refused(fn, good, changes):
    for status, change in changes:
        args = list(good)
        for k, v in change.items():
            args[k] = v
        assert fn(*args) == status, (status, change, nf.nf_last_error())
        assert nf.nf_last_error()


def test_lookup():
    fn = nf.load().nf_embedding_lookup
    #       table type ld V d ids bytes T scale out type ld stream
    good = [FAKE, 0, 64, 100, 64, FAKE, 8, 10, F(1.0), FAKE, 1, 64, None]
    refused(fn, good, [
        (INVALID, {1: 3}), (INVALID, {10: -1}), (INVALID, {2: 63}), (INVALID, {11: 63}), (INVALID, {3: -1}),
        (INVALID, {4: -1}), (INVALID, {4: (1 << 24) + 1, 2: BIG, 11: BIG}), (INVALID, {6: 2}), (INVALID, {7: -1}),
        (INVALID, {7: 1 << 31}), (INVALID, {0: None}), (INVALID, {5: None}), (INVALID, {9: None}),
        (ALIGN, {0: ODD}), (ALIGN, {5: P(0x1004)}), (ALIGN, {9: ODD})])
    for k in (4, 7):  # nothing to do
        args = list(good)
        args[k] = 0
        assert fn(*args) == nf.NF_OK


def test_grad():
    fn = nf.load().nf_embedding_grad
    W, T, V, d = 2, 100, 50, 64
    need = nf.nf_embedding_workspace_bytes(W, T, V, d)
    assert need > 0
    #       dy type ld stride ids bytes ids_stride W T V d scale padding accumulate grads worker_stride ws bytes stream
    good = [FAKE, 0, d, T * d, FAKE, 4, T, W, T, V, d, F(1.0), -1, 0, FAKE, V * d, WS, need, None]
    refused(fn, good, [
        (INVALID, {1: 7}), (INVALID, {2: d - 1}), (INVALID, {3: T * d - 1}), (INVALID, {5: 1}), (INVALID, {6: T - 1}),
        (INVALID, {7: 0}), (INVALID, {7: 256}), (INVALID, {8: -1}), (INVALID, {8: (1 << 24) + 1}), (INVALID, {9: -1}),
        (INVALID, {9: 1 << 31}), (INVALID, {10: -1}), (INVALID, {10: (1 << 24) + 1}), (INVALID, {13: 2}),
        (INVALID, {15: V * d - 1}), (INVALID, {0: None}), (INVALID, {4: None}), (INVALID, {14: None}),
        (ALIGN, {0: ODD}), (ALIGN, {4: P(0x1002)}), (ALIGN, {14: P(0x1002)}), (ALIGN, {16: P(0x100010)}),
        (WORKSPACE, {17: need - 1}), (WORKSPACE, {16: None})])
    for k in (9, 10):  # no table: nothing to do
        args = list(good)
        args[k] = 0
        assert fn(*args) == nf.NF_OK
    for bad in ((0, T, V, d), (W, -1, V, d), (W, T, -1, d), (W, T, V, -1), (W, T, 1 << 31, d)):
        assert nf.nf_embedding_workspace_bytes(*bad) == 0


def test_orthogonal():
    lib = nf.load()
    how = nf.orthogonal()
    ref = ctypes.byref(how)
    need = nf.nf_orthogonal_workspace_bytes(40, 30, 2, how)
    assert need > 0
    split = nf.orthogonal(products=nf.NF_PRODUCTS_SPLIT)  # (a short side of at most 64 always takes these products)
    assert nf.nf_orthogonal_workspace_bytes(40, 30, 2, split) == need
    assert nf.nf_orthogonal_workspace_bytes(300, 200, 2, split) > nf.nf_orthogonal_workspace_bytes(300, 200, 2, how) > 0

    def params(**kw):
        p = nf.orthogonal()
        for k, v in kw.items():
            if k == "coef":
                p.coef[2][1] = v
            else:
                setattr(p, k, v)
        return ctypes.byref(p)

    bad_params = [params(products=2), params(steps=0), params(steps=13), params(eps=-1.0), params(eps=float("inf")),
                  params(eps=float("nan")), params(coef=float("nan")), params(coef=float("inf")), None]
    #       src type ld stride dst type ld stride rows cols batch params ws bytes stream
    good = [FAKE, 0, 30, 1200, FAKE, 1, 30, 1200, 40, 30, 2, ref, WS, need, None]
    refused(lib.nf_orthogonalize, good, [(INVALID, {11: p}) for p in bad_params] + [
        (INVALID, {1: 3}), (INVALID, {5: -1}), (INVALID, {2: 29}), (INVALID, {3: 1199}), (INVALID, {6: 29}),
        (INVALID, {7: 1199}), (INVALID, {8: -1}), (INVALID, {9: -1}), (INVALID, {10: -1}), (INVALID, {0: None}),
        (INVALID, {4: None}), (ALIGN, {0: P(0x1002)}), (ALIGN, {4: ODD}), (ALIGN, {12: P(0x100010)}),
        (UNSUPPORTED, {8: (1 << 17) + 1, 3: BIG, 7: BIG}),
        (UNSUPPORTED, {9: (1 << 17) + 1, 2: BIG, 3: BIG, 6: BIG, 7: BIG}),
        (UNSUPPORTED, {10: 65536}), (WORKSPACE, {13: need - 1}), (WORKSPACE, {12: None})])
    for k in (8, 9, 10):
        args = list(good)
        args[k] = 0
        assert lib.nf_orthogonalize(*args) == nf.NF_OK
    for p in bad_params[:-1]:
        assert lib.nf_orthogonal_workspace_bytes(40, 30, 2, p) == 0

    step = nf.matrix_step(0.1)
    #       grad type ld stride mom ld stride weight type ld stride rows cols batch step params ws bytes stream
    good = [FAKE, 0, 30, 1200, FAKE, 30, 1200, FAKE, 1, 30, 1200, 40, 30, 2, ctypes.byref(step), ref, WS, need, None]
    steps = []
    for k in ("lr", "momentum", "weight_decay", "scale"):
        s = nf.matrix_step(0.1)
        setattr(s, k, float("nan"))
        steps.append(ctypes.byref(s))
    s = nf.matrix_step(0.1)
    s.nesterov = 2
    refused(lib.nf_orthogonal_update, good, [(INVALID, {14: x}) for x in steps + [ctypes.byref(s), None]] +
            [(INVALID, {15: p}) for p in bad_params] + [
        (INVALID, {1: 3}), (INVALID, {8: 3}), (INVALID, {2: 29}), (INVALID, {5: 29}), (INVALID, {6: 1199}),
        (INVALID, {9: 29}), (INVALID, {10: 1199}), (INVALID, {0: None}), (INVALID, {4: None}), (INVALID, {7: None}),
        (ALIGN, {4: P(0x1002)}), (ALIGN, {7: ODD}), (UNSUPPORTED, {13: 65536}), (WORKSPACE, {17: need - 1})])


def test_binding():
    f, ws = torch.zeros(4, 6), torch.zeros(256, dtype=torch.uint8)
    how = nf.orthogonal()
    for call in (
            lambda: nf.nf_orthogonalize(f, f, how, ws),                                         # not on a device
            lambda: nf.nf_orthogonalize(f.t(), f.t(), how, ws),                                 # columns adjacent
            lambda: nf.nf_orthogonalize(f[0], f[0], how, ws),                                   # a vector
            lambda: nf.nf_orthogonal_update(f, f.half(), f, nf.matrix_step(0.1), how, ws),      # momentum's type
            lambda: nf.nf_embedding_lookup(f, torch.zeros(3, dtype=torch.int64), f[:3]),        # not on a device
            lambda: nf.nf_embedding_lookup(f.t(), torch.zeros(3, dtype=torch.int64), f[:3]),
            lambda: nf.nf_embedding_grad(f[None], torch.zeros(1, 4, dtype=torch.int64), f[:1], 0, 1, ws),
            lambda: nf.orthogonal(steps=3, coef=[(1.0, 0.0, 0.0)] * 2)):
        with pytest.raises(ValueError):
            call()
