"""Which product kernels a call runs (no GPU needed): the sizes that the GPU tests run reach all of them."""
import ctypes

import pytest

import paper_2606_25759_amd as nf
from tests.orthogonal_sizes import BF16, F32, SIZES, SINGLE, SPLIT, every_kernel, kernels_of


def test_every_kernel_is_reached():
    reached = set().union(*(kernels_of(*size) for size in SIZES))
    assert len(every_kernel()) == 28
    assert reached == every_kernel()


def test_tiles_differ_within_a_call():
    """One call whose products take tiles of 256, 128 and 64."""
    i = nf.nf_orthogonal_path(500, 4000, 8, nf.orthogonal())
    assert (i.step_tile, i.gram_tile, i.poly_tile) == (256, 128, 64) and i.shares > 1
    assert (8, 500, 4000, SINGLE, BF16) in SIZES


def test_path():
    def path(rows, cols, batch, products, dst_type, steps=5):
        i = nf.nf_orthogonal_path(rows, cols, batch, nf.orthogonal(products=products, steps=steps), dst_type)
        return [getattr(i, k) for k, _ in i._fields_]

    # the products of the largest kind: tiles of 256, a Gram matrix, a polynomial and a product with X a step
    assert path(2048, 2048, 24, SINGLE, BF16) == [0, 256, 256, 256, 1, 5, 5]
    assert path(2048, 2048, 24, SINGLE, BF16) == path(2048, 2048, 24, SINGLE, F32)
    # a short side of at most 64: always pairs, two rounds (three steps and two), nothing but BOTH between them
    for products in (SINGLE, SPLIT):
        assert path(64, 576, 3, products, BF16)[0::5] == [1, 2] and path(64, 576, 3, products, BF16)[6] == 0
    # an FP32 result of pairs goes step by step; into 16 bits a long side takes three steps and two at once
    assert path(257, 449, 40, SPLIT, F32)[5:] == [5, 5]
    assert path(257, 449, 40, SPLIT, BF16)[5:] == [2, 14]
    for empty in ((0, 5, 1), (5, 0, 1), (5, 5, 0)):
        assert path(*empty, SINGLE, BF16) == [0] * 7


def test_the_schedule_decides_the_form():
    """Steps are taken at once only where the call's own steps gain by it; room for it is there whatever they are."""
    long_sides = [(40, 257, 449, SPLIT), (20, 769, 65, SPLIT), (12, 100, 4000, SINGLE), (3, 6001, 150, SINGLE),
                  (25, 3456, 143, SINGLE), (8, 768, 16_384, SINGLE), (4, 1024, 32_768, SINGLE)]
    steep = (7.5, -10.0, 3.6)  # two such steps grow by more than may be taken at once
    for batch, m, n, products in long_sides:
        def path(how):
            i = nf.nf_orthogonal_path(m, n, batch, how)
            return i.split, i.rounds, i.squares

        one_by_one = int(products == SPLIT)
        assert path(nf.orthogonal(products=products)) == (1, 2, 14)
        assert path(nf.orthogonal(products=products, steps=1)) == (one_by_one, 1, 1)
        assert path(nf.orthogonal(products=products, steps=4, coef=steep)) == (one_by_one, 4, 4)
        need = {nf.nf_orthogonal_workspace_bytes(m, n, batch, how)
                for how in (nf.orthogonal(products=products, steps=s, coef=c)
                            for s in range(1, 13) for c in (steep, (2.0, -1.5, 0.5), (3.4445, -4.7750, 2.0315)))}
        assert len(need) == 1


def test_refusals():
    fn, how, info = nf.load().nf_orthogonal_path, nf.orthogonal(), nf.nf_orthogonal_path_info()
    good = [40, 30, 2, ctypes.byref(how), 1, ctypes.byref(info)]
    assert fn(*good) == nf.NF_OK and info.step_tile == 64
    for status, k, v in ((nf.NF_ERR_INVALID_ARG, 0, -1), (nf.NF_ERR_INVALID_ARG, 1, -1), (nf.NF_ERR_INVALID_ARG, 2, -1),
                         (nf.NF_ERR_INVALID_ARG, 3, None), (nf.NF_ERR_INVALID_ARG, 4, 3),
                         (nf.NF_ERR_INVALID_ARG, 5, None), (nf.NF_ERR_UNSUPPORTED, 2, 65536)):
        bad = list(good)
        bad[k] = v
        assert fn(*bad) == status
    with pytest.raises(nf.NFError):
        nf.nf_orthogonal_path(40, 30, 2, nf.orthogonal(steps=13))
