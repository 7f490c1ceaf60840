"""Sizes that between them run every product kernel of the orthogonalisation, and which kernels a size runs.

A kernel is (tile, split operands, epilogue, tile's k shared by several blocks).
"""
import paper_2606_25759_amd as nf

SINGLE, SPLIT = nf.NF_PRODUCTS_SINGLE, nf.NF_PRODUCTS_SPLIT
F32, BF16 = nf.NF_TYPE_F32, nf.NF_TYPE_BF16

# batch, rows, cols, products, type of the result; sides that are no multiple of the tile, wide and tall
SIZES = [
    (3, 60, 40, SINGLE, BF16),
    (2, 64, 700, SINGLE, BF16),
    (2, 65, 66, SINGLE, BF16),
    (2, 190, 130, SINGLE, BF16),
    (5, 513, 1100, SINGLE, BF16),
    (30, 449, 385, SINGLE, BF16),
    (30, 769, 65, SINGLE, BF16),
    (48, 641, 200, SINGLE, BF16),
    (16, 769, 769, SINGLE, BF16),
    (8, 500, 4000, SINGLE, BF16),
    (3, 2100, 1900, SINGLE, BF16),
    (2, 66, 65, SPLIT, F32),
    (2, 130, 190, SPLIT, F32),
    (16, 385, 385, SPLIT, F32),
    (8, 600, 385, SPLIT, F32),
    (8, 385, 600, SPLIT, BF16),
    (40, 257, 449, SPLIT, BF16),
    (20, 769, 65, SPLIT, F32),
    (20, 769, 65, SPLIT, BF16),
]


def kernels_of(batch, rows, cols, products, dst_type, steps=5):
    how = nf.orthogonal(products=products, steps=steps)
    i = nf.nf_orthogonal_path(rows, cols, batch, how, dst_type)
    split, shared = bool(i.split), i.shares > 1
    if min(rows, cols) <= 64:
        got = {(i.gram_tile, split, "BOTH", shared)}
    else:
        got = {(i.gram_tile, split, "GRAM", shared), (i.poly_tile, split, "POLY", False)}
        if i.squares > i.rounds:
            got.add((i.poly_tile, split, "MULT", False))
    got.add((i.step_tile, split, "LAST", False))
    if i.rounds > 1:
        got.add((i.step_tile, split, "STEP", False))
    return got


def every_kernel():
    one = [(t, s) for s, most in ((False, 256), (True, 128)) for t in (64, 128, 256) if t <= most]
    got = {(t, s, e, False) for t, s in one for e in ("GRAM", "POLY", "STEP", "LAST")}
    got |= {(t, s, "GRAM", True) for t, s in one if t < 256}
    got |= {(t, True, "MULT", False) for t in (64, 128)}
    return got | {(64, True, "BOTH", shared) for shared in (False, True)}
