"""Which tiles and shares FP32 takes where the rules for 16 bits are not its own, and that the workspace, whose query names no
type, holds the shares of every type (no GPU needed)."""
import random

import paper_2606_25759_amd as nf
from tests import test_gpu_expert_f32 as u
from tests import test_gpu_expert_far_rows as far
from tests.test_expert_paths import CODES, whole

GRAD = nf.NF_EXPERT_GRAD


def path(op, kind, W, T, E, n, k, lengths):
    i = nf.nf_expert_path(op, CODES[kind], W, T, E, n, k, whole(kind, *lengths))
    return i.tile_columns, i.tile_rows, i.direct, i.share


def product(op, kind, W, E, T, n, k, extra=0):
    return path(op, kind, W, T, E, n, k, (n, k, n + extra, k + extra) if op else (k, k + extra))[:3]


def test_f32_shares_by_its_own_cost():
    """A token of FP32 takes six to eight times as long as one of 16 bits, which its plan has to know."""
    for W, E, T, n, k in u.F32_SHARED:
        assert path(GRAD, "f32", W, T, E, n, k, (n, k))[3] > 0, (W, E, T, n, k)
    for W, E, T, n, k in u.F32_SHARED[:3]:
        assert path(GRAD, "bf16", W, T, E, n, k, (n, k))[3] == 0
    # one block a CU already, sizes alike: 49 us, 71 with shares of 384
    assert path(GRAD, "f32", 1, 2048, 4, 1024, 1024, (1024, 1024))[3] == 0


def test_f32_narrow_results():
    """Long sums into few columns take tiles of 32, though there are many of 128 x 32."""
    for op, case in ((0, (1, 3, 22_635, 19, 3000)), (1, (1, 1, 3326, 3762, 80)), (1, (1, 23, 3811, 3712, 24)),
                     (0, (1, 1, 4126, 24, 2688))):
        assert product(op, "f32", *case)[:2] == (32, 32), case
    assert product(0, "f32", 1, 32, 32_768, 4096, 2048)[:2] == (128, 128)


def test_workspace_holds_every_share():
    """The query names no type: what it says has to do for any, at any alignment."""
    rng = random.Random(3)
    seen = 0
    for _ in range(3000):
        W, E, n, k = rng.choice([1, 1, 2, 8]), int(64 ** rng.random() * rng.choice([1, 1, 20])), rng.randint(1, 2000), rng.randint(1, 2000)
        T = int(32_768 ** rng.random()) * rng.choice([1, 1, 8])
        need = nf.nf_expert_grad_workspace_bytes(W, T, E, n, k)
        tiles = -(-n // 128) * -(-k // 128)
        for kind in CODES:
            for at_once in (0, 1):
                i = nf.nf_expert_path(GRAD, CODES[kind], W, T, E, n, k, at_once)
                if i.share:
                    assert i.tile_columns == i.tile_rows == 128 and i.share < T
                    assert need >= W * (T // i.share + E) * tiles * 128 * 128 * 4
                    seen += 1
        assert need <= 1024 * 128 * 128 * 4
    assert seen > 500


def test_far_rows():
    """The query does not know of far rows; these sizes take the same tile either way."""
    tiles = [path(int(back), "f32", 1, T, 1, n, k, (1,))[:2] for T, n, k, back in far.MATRICES]
    assert tiles == 2 * [(32, 32), (128, 32), (128, 128)]
    assert path(GRAD, "f32", 1, 500, 1, 70, 96, (1,))[3] > 0 and path(GRAD, "f32", 1, 60, 1, 100, 72, (1,))[3] == 0
