"""What the sizes of the GPU tests reach: every product kernel with results of 16 bits and of 32, every one with more experts
than lanes, and shared gradients of them (no GPU needed)."""
import paper_2606_25759_amd as nf
from tests import test_gpu_expert as t
from tests import test_gpu_expert_f32 as f
from tests import test_gpu_expert_kernels as u
from tests.test_expert_f32_paths import path, product
from tests.test_expert_paths import CODES, OPS

GRAD = nf.NF_EXPERT_GRAD


def products():
    """(kernel, bytes of a result, more than 64 experts) of every product that the tests run."""
    found = set()

    def add(op, kind, out, case):
        W, E, T, n, k, extra = case
        found.add((op, kind, *product(op, kind, *case), 4 if out == "f32" else 2, E > 64))

    for op in OPS:
        for kind, out in (("bf16", "bf16"), ("f16", "f32"), ("f32", "f32"), ("f32", "f16"), ("bf16", "f16")):
            for case in t.PRODUCTS:
                add(op, kind, out, case)
        for kind, out in [(k, "f32") for k in CODES] + [("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16")]:
            for case in t.OTHER_PRODUCTS:
                add(op, kind, out, case)
        for kind, out in (("f32", "f32"), ("f32", "f16"), ("bf16", "f32")):
            for W, E, T, n, k, extra in f.NARROW_RESULTS:
                add(op, kind, out, (W, E, T, *((k, n) if op else (n, k)), extra))
        for kind, out in (("bf16", "bf16"), ("f16", "f32"), ("f32", "f32")):
            for W, E, T, n, k, extra in u.MANY_EXPERTS:
                add(op, kind, out, (W, E, T, *((k, n) if op else (n, k)), extra))
    for W, E, T, n, k, back in t.WIDE_PRODUCTS:
        for kind, out in (("bf16", "bf16"), ("f16", "f32")):
            add(OPS[back], kind, out, (W, E, T, n, k, 0))
    for W, E, T, n, k, back in t.F32_PRODUCTS:
        for out in ("f32", "bf16"):
            add(OPS[back], "f32", out, (W, E, T, n, k, 0))
    return found


def test_results_of_every_width():
    got = {p[:6] for p in products()}
    for op in OPS:
        for kind in CODES:
            for tile in ((32, 32), (128, 32), (128, 128)):
                for direct in (0, 1):
                    for size in (2, 4):
                        assert (op, kind, *tile, direct, size) in got, (op, kind, tile, direct, size)
        assert {(op, "bf16", 256, 256, 1, 2), (op, "f16", 256, 256, 1, 4)} <= got


def test_more_experts_than_lanes():
    got = {p[:5] for p in products() if p[6]}
    for op in OPS:
        for kind in CODES:
            for tile in ((32, 32), (128, 32), (128, 128)):
                for direct in (0, 1):
                    assert (op, kind, *tile, direct) in got, (op, kind, tile, direct)
        assert {(op, "bf16", 256, 256, 1), (op, "f16", 256, 256, 1)} <= got
    for kind in CODES:
        for W, E, T, n, k in u.MANY_SHARED:
            assert E > 64 and path(GRAD, kind, W, T, E, n, k, (n, k))[3] > 0
        for W, E, T, n, k in u.MANY_WIDE if kind != "f32" else []:
            assert E > 64 and path(GRAD, kind, W, T, E, n, k, (n, k))[:2] == (256, 256)
        for W, E, T, n, k in u.MANY_GRADS:
            assert E > 64 and path(GRAD, kind, W, T, E, n, k, (n, k))[:2] == (128, 128)
    # as many tiles an expert as the order by length asks for, and fewer
    assert {-(-n // 256) * -(-k // 256) >= 16 for _, _, _, n, k in u.MANY_WIDE} == {True, False}
