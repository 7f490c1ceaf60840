"""The operators on either side of the bucket reducer, as cases that can be measured.

Each case is one pass through one operator (`what`):

  lookup   embedding lookup with scaling: T tokens' rows of a V x d table
  embgrad  its gradient: a dense V x d FP32 segment of each of W workers' gradient rows, the rows of one token
           summed in token order; `accumulate` adds to what the rows hold
  ortho    a batch of matrices (m x n) orthogonalised by Newton-Schulz products
  update   the step around it for a batch of weight matrices: momentum in, orthogonalised, weights out

With `own` false, run() computes them in elementary torch operations in 32 bits; with it true, by the library.

Matrices of a batch lie `gap` elements apart in one flat buffer, as one kind of parameter does in the reducer's
output; gradients are a decaying spectrum over an eighth of the rank with noise below it.  Token ids are skewed
(rank r about as often as 1 / r) or even; where a batch is padded (`pad`), one token in eight is -1: no token.
"""
import math
import random

import torch

own = False

DEV = "cuda"
STEPS, COEF, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
LR, MU, DECAY = 0.02, 0.95, 0.01
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # a short prompt's tokens from an FP32 table to BF16 activations: all latency
        dict(name="lookup_64", what="lookup", T=64, V=50_257, d=1024, table="f32", out="bf16", ids="i64", skew=True,
             pad=False),
        # the tokens of a 1.3B-parameter decoder's step: 16 sequences of 2,048
        dict(name="lookup_32k", what="lookup", T=32_768, V=50_257, d=2048, table="f32", out="bf16", ids="i64",
             skew=True, pad=False),
        # the position table of a small image model: four workers, every row hit, all latency
        dict(name="embgrad_w4_197", what="embgrad", W=4, T=197, V=1_970, d=768, dy="f32", ids="i64", skew=False,
             pad=False, accumulate=False, lead=0),
        # one worker of a 1.3B-parameter decoder: 8,192 tokens into the whole table
        dict(name="embgrad_w1_8k", what="embgrad", W=1, T=8_192, V=50_257, d=2048, dy="bf16", ids="i64", skew=True,
             pad=False, accumulate=False, lead=0),
        # sixteen workers' rows on one GPU, width 1024: the largest table gradient
        dict(name="embgrad_w16_2k", what="embgrad", W=16, T=2_048, V=50_257, d=1024, dy="bf16", ids="i64", skew=True,
             pad=True, accumulate=False, lead=4_096),
        # a second micro-batch added to the first, odd width and an odd place in the row
        dict(name="embgrad_odd_add", what="embgrad", W=2, T=30_011, V=10_007, d=515, dy="f16", ids="i32", skew=True,
             pad=False, accumulate=True, lead=517),
        # a residual stage's three 3x3 convolutions as matrices: all latency
        dict(name="ortho_conv_64", what="ortho", batch=3, m=64, n=576, src="f32", dst="bf16", gap=64),
        # an attention projection of width 768 in twelve blocks
        dict(name="ortho_12x768", what="ortho", batch=12, m=768, n=768, src="f32", dst="bf16", gap=768),
        # odd sizes, in and out in FP32
        dict(name="ortho_odd_f32", what="ortho", batch=1, m=1_601, n=1_000, src="f32", dst="f32", gap=0),
        # the attention projections of a 1.3B-parameter decoder's 24 blocks: the largest
        dict(name="ortho_24x2048", what="ortho", batch=24, m=2_048, n=2_048, src="f32", dst="bf16", gap=2_048),
        # a convolution of 256 channels stepped by itself, FP32 weights
        dict(name="update_conv_256", what="update", batch=1, m=256, n=2_304, grad="f32", weight="f32", gap=0),
        # one MLP matrix of four decoder blocks of width 2048, BF16 weights
        dict(name="update_4x8192", what="update", batch=4, m=8_192, n=2_048, grad="f32", weight="bf16", gap=2_048),
    ]


MOST_FLOPS = 5e12   # of a drawn case's products at most, every one in full
MOST_BYTES = 3.3e9  # of a drawn table gradient at most


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _size(rng, lo, hi):
    """A size over the range: round, ragged or odd."""
    k = int(_log(rng, lo, hi))
    unit = rng.choice([1, 1, 8, 64, 128])
    k = max(lo, k // unit * unit) if k >= 2 * unit else k
    return k + 1 if k == 3072 else k


def draw(rng):
    what = rng.choice(["lookup", "embgrad", "embgrad", "ortho", "ortho", "update"])
    if what in ("lookup", "embgrad"):
        d, V = _size(rng, 16, 4_096), int(_log(rng, 200, 60_000))
        skew, ids = rng.random() < 0.7, rng.choice(["i64", "i32"])
        pad = rng.random() < 0.3
        if what == "lookup":
            return dict(what=what, T=int(_log(rng, 1, 40_000)), V=V, d=d, table=rng.choice(list(TYPES)),
                        out=rng.choice(list(TYPES)), ids=ids, skew=skew, pad=pad)
        W = rng.choice([1, 1, 2, rng.randint(2, 16)])
        d = max(8, min(d, int(MOST_BYTES / 4 / W / V)))
        T = int(_log(rng, 1, min(70_000, 3e8 / W / d)))
        return dict(what=what, W=W, T=T, V=V, d=d, dy=rng.choice(list(TYPES)), ids=ids, skew=skew, pad=pad,
                    accumulate=rng.random() < 0.3,
                    lead=rng.choice([0, 0, 4 * rng.randint(1, 5_000), rng.randint(1, 5_000)]))
    m, n = _size(rng, 16, 4_096), _size(rng, 16, 8_192)
    if rng.random() < 0.5:
        m, n = n, m
    one = STEPS * (4 * min(m, n) * m * n + 2 * min(m, n) ** 3)
    batch = max(1, min(48, int(_log(rng, 1, 48.9)), int(MOST_FLOPS / one), int(3e8 / m / n)))
    gap = rng.choice([0, 0, n, rng.randint(1, 4_000)])
    if what == "ortho":
        return dict(what=what, batch=batch, m=m, n=n, src=rng.choice(["f32", "f32", "bf16", "f16"]),
                    dst=rng.choice(["bf16", "bf16", "f16", "f32"]), gap=gap)
    return dict(what=what, batch=batch, m=m, n=n, grad=rng.choice(["f32", "f32", "bf16"]),
                weight=rng.choice(["f32", "bf16"]), gap=gap)


def _flops(m, n):
    """Multiply-adds, times two, that the steps need for one matrix: of a symmetric product half, and with the
    powers applied to X step by step or, for a long side, to the Gram matrix first and X once."""
    m, n = min(m, n), max(m, n)
    return min(STEPS * (3 * m * m * n + m ** 3), 3 * m * m * n + (4 * STEPS - 3) * m ** 3)


def work(case):
    size = lambda t: TYPES[t].itemsize  # noqa: E731
    i = 8 if case.get("ids") == "i64" else 4
    if case["what"] == "lookup":
        rows = min(case["T"], case["V"])  # a row that many tokens share is needed once
        return {"bytes": case["T"] * (i + case["d"] * size(case["out"])) + rows * case["d"] * size(case["table"]),
                "flops": case["T"] * case["d"]}
    if case["what"] == "embgrad":
        W, T, V, d = (case[k] for k in ("W", "T", "V", "d"))
        written = 8 * W * min(T, V) * d if case["accumulate"] else 4 * W * V * d
        return {"bytes": W * T * (i + d * size(case["dy"])) + written, "flops": W * T * d}
    m, n, batch = case["m"], case["n"], case["batch"]
    if case["what"] == "ortho":
        moved = size(case["src"]) + size(case["dst"])
    else:
        moved = size(case["grad"]) + 8 + 2 * size(case["weight"])
    return {"bytes": batch * m * n * moved, "flops": batch * _flops(m, n)}


# -------------------------------------------------------------------- inputs

def _ids(g, shape, V, skew, pad, kind):
    u = torch.rand(shape, generator=g, device=DEV)
    rank = (float(V) ** u - 1).clamp(max=V - 1) if skew else u * V
    # the frequent ids lie all over the table, as a vocabulary's do
    ids = (rank.to(torch.int64).clamp(0, V - 1) * 7_919 + 13) % V
    if pad:
        ids = torch.where(torch.rand(shape, generator=g, device=DEV) < 0.125, -1, ids)
    return ids.to(torch.int64 if kind == "i64" else torch.int32)


def _gradients(g, batch, m, n, gap, kind):
    """`batch` matrices in one flat buffer, and the view of them."""
    flat = torch.randn(batch * (m * n + gap), generator=g, device=DEV)
    view = flat.as_strided((batch, m, n), (m * n + gap, n, 1))
    r = max(1, min(m, n) // 8)
    s = torch.logspace(0, -2, r, device=DEV)
    left = torch.randn(batch, m, r, generator=g, device=DEV) * s
    right = torch.randn(batch, r, n, generator=g, device=DEV)
    view.mul_(0.01 * math.sqrt(r)).add_(left @ right).mul_(1e-3)
    flat = flat.to(TYPES[kind])
    return flat.as_strided((batch, m, n), (m * n + gap, n, 1))


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case)
    if case["what"] == "lookup":
        s["table"] = (torch.randn(case["V"], case["d"], generator=g, device=DEV) * 0.02).to(TYPES[case["table"]])
        s["ids"] = _ids(g, (case["T"],), case["V"], case["skew"], case["pad"], case["ids"])
        s["out"] = torch.empty(case["T"], case["d"], dtype=TYPES[case["out"]], device=DEV)
        s["scale"] = math.sqrt(case["d"])
    elif case["what"] == "embgrad":
        W, T, V, d = (case[k] for k in ("W", "T", "V", "d"))
        s["dy"] = (torch.randn(W, T, d, generator=g, device=DEV) * 1e-3).to(TYPES[case["dy"]])
        s["ids"] = _ids(g, (W, T), V, case["skew"], case["pad"], case["ids"])
        stride = (case["lead"] + V * d + 63) // 64 * 64
        # the workers' rows; what is accumulated onto is the gradient of the micro-batch before
        s["rows"] = torch.randn(W, stride, generator=g, device=DEV) * 1e-3 if case["accumulate"] else \
            torch.empty(W, stride, device=DEV)
        s["segment"] = s["rows"][:, case["lead"]:case["lead"] + V * d].unflatten(1, (V, d))
        s["scale"] = math.sqrt(d)
    elif case["what"] == "ortho":
        s["src"] = _gradients(g, case["batch"], case["m"], case["n"], case["gap"], case["src"])
        s["dst"] = torch.empty(case["batch"], case["m"], case["n"], dtype=TYPES[case["dst"]], device=DEV)
    else:
        size = (case["batch"], case["m"], case["n"])
        s["grad"] = _gradients(g, *size, case["gap"], case["grad"])
        s["momentum"] = _gradients(g, *size, 0, "f32") * 5
        s["weight"] = (torch.randn(size, generator=g, device=DEV) * 0.02).to(TYPES[case["weight"]])
        s["scale"] = math.sqrt(max(1.0, case["m"] / case["n"]))
    return s


# ------------------------------------------------------------------ the pass

def run(state):
    return (_library if own else _plain)(state)


def _workspace(nf, state, size):
    """The workspace that a program keeps from step to step."""
    if "ws" not in state:
        state["ws"] = nf.empty_workspace(size)
    return state["ws"]


def _library(s):
    import paper_2606_25759_amd as nf

    if s["what"] == "lookup":
        nf.nf_embedding_lookup(s["table"], s["ids"], s["out"], scale=s["scale"])
        return s["out"]
    if s["what"] == "embgrad":
        ws = _workspace(nf, s, nf.nf_embedding_workspace_bytes(s["W"], s["T"], s["V"], s["d"]))
        nf.nf_embedding_grad(s["dy"], s["ids"], s["rows"], s["lead"], s["V"], ws, scale=s["scale"],
                             accumulate=s["accumulate"])
        return s["segment"]
    # BF16 results (8 bits) from products of 11-bit operands, FP16 and FP32 results from products of 22-bit ones
    fine = (s["dst"] if s["what"] == "ortho" else s["weight"]).dtype != torch.bfloat16
    how = nf.orthogonal(products=nf.NF_PRODUCTS_SPLIT if fine else nf.NF_PRODUCTS_SINGLE, steps=STEPS, coef=COEF,
                        eps=EPS)
    ws = _workspace(nf, s, nf.nf_orthogonal_workspace_bytes(s["m"], s["n"], s["batch"], how))
    if s["what"] == "ortho":
        nf.nf_orthogonalize(s["src"], s["dst"], how, ws)
        return s["dst"]
    step = nf.matrix_step(lr=LR, momentum=MU, nesterov=True, weight_decay=DECAY, scale=s["scale"])
    nf.nf_orthogonal_update(s["grad"], s["momentum"], s["weight"], step, how, ws)
    return s["momentum"], s["weight"]


def _newton_schulz(u):
    a, b, c = COEF
    x = u / (u.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    for _ in range(STEPS):
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(1, 2) if tall else x


def _plain(s):
    if s["what"] == "lookup":
        ids = s["ids"].to(torch.int64)
        return (s["table"][ids.clamp(min=0)].float() * (s["scale"] * (ids >= 0))[:, None]).to(s["out"].dtype)
    if s["what"] == "embgrad":
        W, V, d = s["W"], s["V"], s["d"]
        # what belongs to no token is summed into a row of its own, past the last worker's
        row = s["ids"].to(torch.int64)
        row = torch.where(row >= 0, row + V * torch.arange(W, device=DEV)[:, None], W * V)
        total = torch.zeros(W * V + 1, d, device=DEV)
        total.index_add_(0, row.reshape(-1), s["dy"].float().reshape(-1, d))
        total = (total[:-1] * s["scale"]).view(W, V, d)
        if s["accumulate"]:
            s["segment"].add_(total)
        else:
            s["segment"].copy_(total)
        return s["segment"]
    if s["what"] == "ortho":
        return _newton_schulz(s["src"].float()).contiguous().to(s["dst"].dtype)
    grad, m, w = s["grad"].float(), s["momentum"], s["weight"]
    m.mul_(MU).add_(grad)
    x = _newton_schulz(grad + MU * m)
    w.copy_(w.float() * (1 - LR * DECAY) - LR * s["scale"] * x)
    return m, w


# ------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["what"] == "lookup":
        out = torch.zeros(case["T"], case["d"], dtype=torch.float64, device=DEV)
        at = torch.nonzero(s["ids"] >= 0).flatten()
        out[at] = s["table"].index_select(0, s["ids"][at].to(torch.int64)).double() * s["scale"]
        return out
    if case["what"] == "embgrad":
        V, d = case["V"], case["d"]
        out = s["segment"].double() if case["accumulate"] else torch.zeros(case["W"], V, d, dtype=torch.float64, device=DEV)
        for w in range(case["W"]):
            at = torch.nonzero(s["ids"][w] >= 0).flatten()
            out[w].index_add_(0, s["ids"][w][at].to(torch.int64), s["dy"][w][at].double() * s["scale"])
        return out
    if case["what"] == "ortho":
        return torch.stack([_orthogonal64(x.double()) for x in s["src"]])
    g, m = s["grad"].double(), s["momentum"].double()
    m = MU * m + g
    step = torch.stack([_orthogonal64(x) for x in g + MU * m])
    return m, s["weight"].double() * (1 - LR * DECAY) - (LR * s["scale"]) * step


def _orthogonal64(u):
    """a X + X (b C + c C C) with C = X^T X on the side that is shorter, one matrix at a time."""
    a, b, c = COEF
    if u.shape[0] < u.shape[1]:
        return _orthogonal64(u.T.contiguous()).T.contiguous()
    x = u / (torch.linalg.vector_norm(u) + EPS)
    one = torch.eye(u.shape[1], dtype=torch.float64, device=DEV)
    for _ in range(STEPS):
        cc = x.T.contiguous() @ x
        x = x @ (a * one + cc @ (b * one + c * cc))
    return x
