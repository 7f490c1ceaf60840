"""Results that share elements with operands are refused, as far as their layouts show it (no GPU needed); those that only
lie between one another's rows are taken (test_gpu_expert_overlap.py)."""
import pytest

import paper_2606_25759_amd as nf
from tests.test_operator_refusals import INVALID, P

BASE = 0x7000_0000_0000
FAR = 0x7100_0000_0000


def product(x, w, y, W=2, T=10, E=4, n=24, k=40, x_ld=None, x_stride=None, y_ld=None, y_stride=None, w_ld=None,
            w_stride=None, type=1, y_type=1):
    x_ld, y_ld, w_ld = x_ld or k, y_ld or n, w_ld or k
    st = nf.load().nf_expert_product(P(x), type, x_ld, x_stride or T * x_ld, P(w), w_ld, w_stride or n * w_ld, 0,
                                     P(FAR + (1 << 40)), 4, E + 1, W, T, E, n, k, P(y), y_type, y_ld, y_stride or T * y_ld,
                                     None)
    return st, nf.nf_last_error()


X_BYTES = 2 * 10 * 40 * 2  # of the product above
W_BYTES = 4 * 24 * 40 * 2
Y_BYTES = 2 * 10 * 24 * 2


@pytest.mark.parametrize("at", [2, 100, X_BYTES - 2, -2, 2 - Y_BYTES])
def test_product_into_its_rows(at):
    st, why = product(BASE, FAR, BASE + at)
    assert st == INVALID and "shares" in why


@pytest.mark.parametrize("at", [2, 1000, W_BYTES - 2, -2, 2 - Y_BYTES])
def test_product_into_its_matrices(at):
    st, why = product(FAR, BASE, BASE + at)
    assert st == INVALID and "shares" in why


@pytest.mark.parametrize("change,at", [
    # columns 0 to 39 of rows of 64 elements, and y's 24 of the same rows: from column 39, from one before (around the end)
    (dict(x_ld=64, y_ld=64), 2 * 39), (dict(x_ld=64, y_ld=64), 2 * (64 - 23)), (dict(x_ld=64, y_ld=64), -2 * 23),
    (dict(x_ld=64, y_ld=64), 2 * (64 * 19 + 39)), (dict(x_ld=64, y_ld=64), 2 * (-64 * 19 - 23)),
    # y's rows of FP32, the same way apart
    (dict(x_ld=88, y_ld=44, y_type=0), 2 * 38), (dict(x_ld=88, y_ld=44, y_type=0), 2 * (88 - 46)),
    # y in one run of memory, across rows of x that are apart
    (dict(x_ld=4096), 2 * (4096 * 3 - 470)), (dict(x_ld=4096), 2 * (4096 * 19 + 39)),
    # rows of x in one run, across rows of y
    (dict(y_ld=4096), -2 * 4096 * 19), (dict(y_ld=4096), 2 * (799 - 4096)),
    # one row each
    (dict(W=1, T=1, x_ld=99, y_ld=77), 2 * 39), (dict(W=1, T=1), -2 * 23)])
def test_product_between_rows(change, at):
    st, why = product(BASE, FAR, BASE + at, **change)
    assert st == INVALID and "shares" in why


def grad(dy, x, grads, W=2, T=5000, E=2, n=24, k=40, matrix=None, worker=None, type=0):
    need = nf.nf_expert_grad_workspace_bytes(W, T, E, n, k)
    matrix = matrix or n * k
    st = nf.load().nf_expert_grad(P(dy), n, T * n, P(x), k, T * k, type, P(FAR + (1 << 40)), 8, E + 1, W, T, E, n, k, 0,
                                  P(grads), matrix, worker or E * matrix, P(FAR + (1 << 41)), need, None)
    return st, nf.nf_last_error()


DY_BYTES, G_BYTES = 2 * 5000 * 24 * 4, 2 * 2 * 24 * 40 * 4


@pytest.mark.parametrize("at", [0, 4, DY_BYTES - 4, -4, 4 - G_BYTES])
def test_grad_into_its_operands(at):
    for dy, x in ((BASE, FAR), (FAR, BASE)):
        st, why = grad(dy, x, BASE + at)
        assert st == INVALID and "shares" in why
    # matrices that are apart: a worker's second one reaches into x
    st, why = grad(FAR, BASE, BASE + 4 * (40 - (1 << 20)), W=1, matrix=1 << 20)
    assert st == INVALID and "shares" in why
