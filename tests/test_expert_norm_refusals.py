"""Refusals of the expert and norm entry points: an error code before anything is launched (no GPU needed), and the
binding's own checks."""
import ctypes

import pytest
import torch

import paper_2606_25759_amd as nf
from tests.test_operator_refusals import ALIGN, FAKE, INVALID, ODD, UNSUPPORTED, WORKSPACE, WS, P, refused

BIG = 1 << 40
FAR = [1 << 62, (1 << 62) + 1, (1 << 63) - 1, 3 << 60]  # times 9 past 64 bits
OTHER = P(0x2000)


def test_product():
    fn = nf.load().nf_expert_product
    W, T, E, n, k = 2, 10, 4, 24, 40
    #       x type ld stride w ld stride transposed offsets bytes stride W T E n k y type ld stride stream
    good = [FAKE, 1, k, T * k, OTHER, k, n * k, 0, FAKE, 4, E + 1, W, T, E, n, k, P(0x3000), 1, n, T * n, None]
    refused(fn, good, [
        (INVALID, {1: 3}), (INVALID, {17: -1}), (INVALID, {7: 2}), (INVALID, {9: 2}), (INVALID, {2: k - 1}),
        (INVALID, {3: T * k - 1}), (INVALID, {5: k - 1}), (INVALID, {6: n * k - 1}), (INVALID, {10: E}),
        (INVALID, {11: 0}), (INVALID, {11: 256}), (INVALID, {12: -1}), (INVALID, {12: (1 << 24) + 1, 3: BIG, 19: BIG}),
        (INVALID, {13: -1}), (INVALID, {13: 4097}), (INVALID, {14: -1}), (INVALID, {15: -1}),
        (INVALID, {14: (1 << 20) + 1}), (INVALID, {18: n - 1}), (INVALID, {19: T * n - 1}), (INVALID, {0: None}),
        (INVALID, {4: None}), (INVALID, {8: None}), (INVALID, {16: None}), (INVALID, {16: FAKE}), (INVALID, {16: OTHER}),
        (INVALID, {7: 1}),  # x has n columns then, y k
        (ALIGN, {0: ODD}), (ALIGN, {4: ODD}), (ALIGN, {16: ODD}), (ALIGN, {8: P(0x1002)}),
        (ALIGN, {8: P(0x1004), 9: 8}),
        (UNSUPPORTED, {12: 1 << 24, 3: BIG, 19: BIG, 11: 200, 14: 2000, 6: BIG, 18: 2000})])
    refused(fn, good, [(INVALID, {k: ld}) for k in (2, 5, 18) for ld in FAR])
    for change in ({12: 0}, {13: 0}, {14: 0}):  # nothing to do
        args = list(good)
        for i, v in change.items():
            args[i] = v
        assert fn(*args) == nf.NF_OK


def test_grad():
    fn = nf.load().nf_expert_grad
    W, T, E, n, k = 2, 5000, 2, 24, 40
    need = nf.nf_expert_grad_workspace_bytes(W, T, E, n, k)
    assert need > 0
    #       dy ld stride x ld stride type offsets bytes stride W T E n k acc grads matrix worker ws bytes stream
    good = [FAKE, n, T * n, FAKE, k, T * k, 1, FAKE, 8, E + 1, W, T, E, n, k, 0, FAKE, n * k, E * n * k, WS, need, None]
    refused(fn, good, [
        (INVALID, {6: 5}), (INVALID, {8: 0}), (INVALID, {1: n - 1}), (INVALID, {2: T * n - 1}), (INVALID, {4: k - 1}),
        (INVALID, {5: T * k - 1}), (INVALID, {9: E}), (INVALID, {10: 0}), (INVALID, {10: 256}), (INVALID, {11: -1}),
        (INVALID, {11: (1 << 24) + 1, 2: BIG, 5: BIG}), (INVALID, {12: -1}), (INVALID, {12: 4097}), (INVALID, {13: -1}),
        (INVALID, {14: -1}), (INVALID, {14: (1 << 20) + 1}), (INVALID, {15: 2}), (INVALID, {17: n * k - 1}),
        (INVALID, {18: E * n * k - 1}), (INVALID, {0: None}), (INVALID, {3: None}), (INVALID, {7: None}),
        (INVALID, {16: None}), (ALIGN, {0: ODD}), (ALIGN, {3: ODD}), (ALIGN, {16: P(0x1002)}), (ALIGN, {7: P(0x1004)}),
        (ALIGN, {19: P(0x100010)}), (WORKSPACE, {20: need - 1}), (WORKSPACE, {19: None})])
    refused(fn, good, [(INVALID, {k: ld}) for k in (1, 4, 17) for ld in FAR])
    for i in (12, 13, 14):
        args = list(good)
        args[i] = 0
        assert fn(*args) == nf.NF_OK
    for sizes in ((0, T, E, n, k), (W, -1, E, n, k), (W, T, 4097, n, k), (W, T, E, -1, k)):
        assert nf.nf_expert_grad_workspace_bytes(*sizes) == 0


def plan_of(tensors, groups=1):
    plan = nf.nf_norm_plan()
    array = (nf.nf_norm_tensor * max(1, len(tensors)))(*tensors)
    return nf.load().nf_norm_plan_init(array, len(tensors), groups, ctypes.byref(plan)), plan


def tensor(src=0x10000, dst=None, rows=10, cols=20, src_ld=20, dst_ld=20, src_type=0, dst_type=0, group=0):
    return nf.nf_norm_tensor(src, dst, rows, cols, src_ld, dst_ld, src_type, dst_type, group, 0)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(src_type=3)), (INVALID, dict(dst=0x20000, dst_type=9)), (INVALID, dict(group=1)),
    (INVALID, dict(group=-1)), (INVALID, dict(rows=-1)), (INVALID, dict(cols=-1)), (INVALID, dict(src_ld=19)),
    (INVALID, dict(dst=0x20000, dst_ld=19)), (INVALID, dict(src=None)), (ALIGN, dict(src=0x10002)),
    (ALIGN, dict(dst=0x20001, dst_type=1)), (INVALID, dict(src_ld=1 << 60)), (INVALID, dict(rows=1 << 61, src_ld=1 << 5)),
    (INVALID, dict(cols=1 << 62, src_ld=1 << 62)), (UNSUPPORTED, dict(rows=1 << 35, src_ld=24)),
    (INVALID, dict(dst=0x10000, dst_type=1)), (INVALID, dict(dst=0x10004)), (INVALID, dict(dst=0x10000, dst_ld=24))])
def test_plan(status, change):
    st, plan = plan_of([tensor(**change)])
    assert st == status, nf.nf_last_error()
    assert plan.table_bytes == 0 and nf.nf_last_error()


def test_plan_of_tensors_that_share_elements():
    a = dict(dst=0x10000)  # in place: 10 rows of 80 bytes at 0x10000
    left = dict(cols=12, dst=0x10000)
    right = dict(src=0x10000 + 48, cols=8, dst=0x10000 + 48)  # columns 12 to 19 of the same rows
    for tensors, status in (
            ([a, a], INVALID), ([a, dict()], INVALID), ([dict(), dict()], nf.NF_OK), ([left, right], nf.NF_OK),
            ([left, dict(right, src=0x10000 + 44, cols=9, dst=0x10000 + 44)], INVALID),
            ([left, dict(src=0x10000 + 48, cols=8)], nf.NF_OK), ([left, dict(src=0x10000 + 47 * 4)], INVALID),
            ([a, dict(src=0x10000 + 800)], nf.NF_OK), ([a, dict(src=0x10000 + 796)], INVALID),
            ([dict(dst=0x20000), dict(dst=0x20000 + 400)], INVALID), ([dict(dst=0x20000), dict(dst=0x20000 + 800)], nf.NF_OK),
            ([dict(dst=0x20000), dict(src=0x20000)], INVALID), ([a, dict(rows=0)], nf.NF_OK)):
        for order in (tensors, tensors[::-1]):
            st, _ = plan_of([tensor(**t) for t in order])
            assert st == status, (tensors, nf.nf_last_error())


def test_what_is_not_read_may_be_anything():
    """The strides of one row, and those of a place that there is not."""
    for change in (dict(dst_ld=-1), dict(dst_ld=1 << 62, dst_type=77), dict(rows=1, src_ld=-5),
                   dict(rows=1, src_ld=0, dst=0x20000, dst_ld=-7)):
        st, plan = plan_of([tensor(**change)])
        assert st == nf.NF_OK and plan.pieces == 1, change


def test_plan_sizes():
    assert plan_of([])[0] == nf.NF_OK and plan_of([], 0)[0] == nf.NF_OK
    lib = nf.load()
    plan, one = nf.nf_norm_plan(), (nf.nf_norm_tensor * 1)(tensor())
    for args in ((one, -1, 1), (one, (1 << 20) + 1, 1), (one, 1, -1), (one, 1, (1 << 16) + 1), (None, 1, 1)):
        assert lib.nf_norm_plan_init(*args, ctypes.byref(plan)) == INVALID
    assert lib.nf_norm_plan_init(one, 1, 1, None) == INVALID
    # every group has a block, and no more than the card holds beside them
    for groups in (1, 7, 3000):
        st, plan = plan_of([tensor(src=0x10000 + (i << 28), rows=1, cols=40_000_000, group=i % groups) for i in range(9)], groups)
        assert st == nf.NF_OK and groups <= plan.blocks <= 512 + groups and plan.workspace_bytes == 8 * plan.blocks


def test_calls():
    lib = nf.load()
    st, plan = plan_of([tensor(dst=0x20000)])
    ref = ctypes.byref(plan)
    one = (nf.nf_norm_tensor * 1)(tensor(dst=0x20000))
    need = plan.table_bytes
    other = nf.nf_norm_plan.from_buffer_copy(plan)
    other.pieces += 1
    refused(lib.nf_norm_table_init, [one, 1, ref, WS, need, None], [
        (INVALID, {2: None}), (INVALID, {2: ctypes.byref(other)}), (INVALID, {3: None}), (ALIGN, {3: P(0x100010)}),
        (WORKSPACE, {4: need - 1}), (INVALID, {1: 0}), (INVALID, {0: None})])
    ws = plan.workspace_bytes
    bad = nf.nf_norm_plan.from_buffer_copy(plan)
    bad.blocks = 0
    common = [(INVALID, {0: None}), (ALIGN, {0: P(0x100010)}), (INVALID, {1: None}), (INVALID, {1: ctypes.byref(bad)})]
    refused(lib.nf_grad_norm, [WS, ref, FAKE, WS, ws, None], common + [
        (INVALID, {2: None}), (ALIGN, {2: P(0x1002)}), (WORKSPACE, {3: None}), (ALIGN, {3: P(0x100010)}),
        (WORKSPACE, {4: ws - 1})])
    F = ctypes.c_float
    limits = [F(-1.0), F(float("nan")), F(float("inf"))]
    _, reads = plan_of([tensor()])
    refused(lib.nf_grad_clip, [WS, ref, FAKE, F(1.0), F(0.0), None], common + [
        (INVALID, {2: None}), (INVALID, {1: ctypes.byref(reads)})] + [(INVALID, {i: x}) for i in (3, 4) for x in limits])
    refused(lib.nf_grad_norm_clip, [WS, ref, F(1.0), F(0.0), FAKE, WS, ws, None], common + [
        (INVALID, {4: None}), (INVALID, {1: ctypes.byref(reads)}), (WORKSPACE, {6: ws - 1}), (WORKSPACE, {5: None})] +
        [(INVALID, {i: x}) for i in (2, 3) for x in limits])
    empty = plan_of([], 0)[1]
    assert lib.nf_grad_norm(None, ctypes.byref(empty), None, None, 0, None) == nf.NF_OK


def test_binding():
    f, off, ws = torch.zeros(4, 6), torch.zeros(3, dtype=torch.int32), torch.zeros(256, dtype=torch.uint8)
    w = torch.zeros(2, 5, 6)
    for call in (
            lambda: nf.nf_expert_product(f, w, off, f.new_zeros(4, 5)),                   # not on a device
            lambda: nf.nf_expert_product(f, w[0], off, f.new_zeros(4, 5)),                # one matrix
            lambda: nf.nf_expert_product(f.t(), w, off, f.new_zeros(6, 5)),               # columns adjacent
            lambda: nf.nf_expert_grad(f, f, off, torch.zeros(1, 72), 0, ws),              # not on a device
            lambda: nf.norm_plan([f]),                                                    # not on a device
            lambda: nf.norm_plan([f], [f, f]), lambda: nf.norm_plan([f], [f.t()]), lambda: nf.norm_plan([f], groups=[0, 1])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError, match="expanded"):
        nf.binding._parts(torch.zeros(3, 1).expand(3, 4), None, "t")
    parts = nf.binding._parts
    t = torch.zeros(4, 5, 6)
    assert parts(t, None, "t") == (1, 120, 120, 120, [(0, 0)])
    assert parts(t.permute(2, 0, 1), None, "t") == (1, 120, 120, 120, [(0, 0)])
    assert parts(t[:, :, :5], None, "t") == (20, 5, 6, 6, [(0, 0)])
    assert parts(t[:, 1:, :5], None, "t") == (4, 5, 6, 6, [(0, 0), (30, 30), (60, 60), (90, 90)])
    assert parts(t[:, 1:], torch.zeros(4, 4, 6), "t") == (4, 24, 30, 24, [(0, 0)])
    assert parts(torch.zeros(6, 4).t(), torch.zeros(4, 6), "t") == (4, 1, 1, 6, [(4 * i, i) for i in range(6)])
    assert parts(torch.zeros(()), None, "t") == (1, 1, 1, 1, [(0, 0)])
