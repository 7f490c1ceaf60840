"""Row and matrix strides whose product passes 64 bits are refused like any that are too far apart (no GPU needed)."""
import ctypes

import pytest

import paper_2606_25759_amd as nf

P = ctypes.c_void_p
FAKE, WS = P(0x1000), P(0x100000)  # never dereferenced: validation fails first
# times 39 or 99 at least 2^63: wrapped to 64 bits most of them come out small or negative
FAR = [1 << 62, (1 << 62) + 1, (1 << 63) - 1, 3 << 60, 5 << 58]


@pytest.mark.parametrize("ld", FAR)
def test_matrices(ld):
    how, step = nf.orthogonal(), nf.matrix_step(0.1)
    need = nf.nf_orthogonal_workspace_bytes(40, 30, 2, how)
    ref = ctypes.byref(how)
    for src, dst in ((ld, 30), (30, ld)):
        assert nf.load().nf_orthogonalize(FAKE, 0, src, 1 << 40, FAKE, 1, dst, 1 << 40, 40, 30, 2, ref, WS, need,
                                          None) == nf.NF_ERR_INVALID_ARG
    for k in range(3):
        lds = [30] * 3
        lds[k] = ld
        assert nf.load().nf_orthogonal_update(FAKE, 0, lds[0], 1 << 40, FAKE, lds[1], 1 << 40, FAKE, 1, lds[2], 1 << 40,
                                              40, 30, 2, ctypes.byref(step), ref, WS, need,
                                              None) == nf.NF_ERR_INVALID_ARG


@pytest.mark.parametrize("ld", FAR)
@pytest.mark.parametrize("T", [3, 100])
def test_gradient(T, ld):
    W, V, d = 2, 50, 64
    need = nf.nf_embedding_workspace_bytes(W, T, V, d)
    assert nf.load().nf_embedding_grad(FAKE, 0, ld, 1 << 40, FAKE, 4, T, W, T, V, d, ctypes.c_float(1.0), -1, 0, FAKE,
                                       V * d, WS, need, None) == nf.NF_ERR_INVALID_ARG
