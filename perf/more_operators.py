"""A layer of experts and the gradient's norm on either side of the bucket reducer, as cases that can be measured.

Each case is one pass through one operator (`what`):

  product  rows of tokens in expert order times their expert's matrix: y = W_e x, or with `back` y = W_e^T x (the
           gradient of the rows)
  grad     the gradient of the experts' matrices for W workers, straight into their FP32 gradient rows; `accumulate`
           adds to what the rows hold
  norm     the norm of each group of many tensors (a worker's gradients)
  clip     norm, and the tensors scaled by min(1, max_norm / norm) into the worker's FP32 row

With `own` false, run() computes them in elementary torch operations in 32 bits (norms in 64); with it true, by the
library.

Expert e of worker w has the rows [offsets[w][e], offsets[w][e + 1]); sizes are uneven, some experts get none
(`empty`: about that share), and a padded batch (`pad`) has rows behind the last expert's, which no operator touches.
The offsets are on the device; a program that works them out on the host has the sizes there too (`sizes`), which the
plain form goes by.
"""
import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # a handful of tokens through a small layer of experts: all latency
        dict(name="product_16", what="product", back=False, W=1, E=8, T=16, n=512, k=256, type="bf16", out="bf16",
             offsets="i32", empty=0.3, pad=False),
        # a few tokens through many experts: every matrix that has a token is read once
        dict(name="product_128_of_64", what="product", back=False, W=1, E=64, T=128, n=1024, k=2048, type="bf16",
             out="bf16", offsets="i32", empty=0.1, pad=False),
        # 16,384 tokens, two experts each, through the first matrices of 32 experts of width 2048: the largest
        dict(name="product_32k", what="product", back=False, W=1, E=32, T=32_768, n=4_096, k=2_048, type="bf16",
             out="bf16", offsets="i32", empty=0.0, pad=False),
        # the gradient of those rows
        dict(name="back_32k", what="product", back=True, W=1, E=32, T=32_768, n=4_096, k=2_048, type="bf16",
             out="bf16", offsets="i32", empty=0.0, pad=False),
        # odd sizes, FP32 out, a padded batch
        dict(name="back_odd", what="product", back=True, W=1, E=7, T=3_001, n=515, k=1_003, type="f16", out="f32",
             offsets="i64", empty=0.2, pad=True),
        # the matrices' gradient of the largest step: 1.07 GB of FP32 into one worker's row
        dict(name="grad_32k", what="grad", W=1, E=32, T=32_768, n=4_096, k=2_048, type="bf16", offsets="i32",
             empty=0.0, pad=False, accumulate=False, lead=0),
        # four workers on one GPU, a second micro-batch added to the first, an odd place in the row
        dict(name="grad_w4_add", what="grad", W=4, E=8, T=2_048, n=1_024, k=512, type="bf16", offsets="i32",
             empty=0.1, pad=True, accumulate=True, lead=517),
        # a long batch through small matrices in FP32
        dict(name="grad_long_f32", what="grad", W=1, E=4, T=30_011, n=256, k=128, type="f32", offsets="i64",
             empty=0.0, pad=False, accumulate=False, lead=4_096),
        # a small model's dozen tensors: all latency
        dict(name="norm_tiny", what="norm", tensors="random", count=12, most=4_096, groups=1, type="f32", shapes=1,
             gap=0, packed=True),
        # sixteen workers' gradients of a 50-layer image model, a norm each
        dict(name="norm_w16_conv", what="norm", tensors="conv", groups=16, type="f32", gap=0, packed=True),
        # one worker's gradients of that model, clipped into its row
        dict(name="clip_conv", what="clip", tensors="conv", groups=1, type="f32", gap=0, packed=False),
        # BF16 gradients of a 1.3B-parameter decoder, clipped into the FP32 row: the largest
        dict(name="clip_1p3b", what="clip", tensors="decoder", groups=1, type="bf16", gap=0, packed=False),
    ]


MOST_FLOPS = 5.4e11   # of a drawn case's products at most
MOST_MATRICES = 2.6e8  # elements of its matrices, or of all workers' gradients of them
MOST_ELEMENTS = 3e8   # of its tensors


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _size(rng, lo, hi):
    """A size over the range: round, ragged or odd."""
    k = int(_log(rng, lo, hi))
    unit = rng.choice([1, 1, 8, 64, 128])
    return max(lo, k // unit * unit) if k >= 2 * unit else k


def draw(rng):
    what = rng.choice(["product", "product", "product", "grad", "grad", "norm", "clip"])
    if what in ("product", "grad"):
        n, k = _size(rng, 16, 4_096), _size(rng, 16, 4_096)
        W = rng.choice([1, 1, 1, rng.randint(2, 8)])
        copies = W if what == "grad" else 1
        E = max(1, min(int(_log(rng, 1, 64.9)), int(MOST_MATRICES / n / k / copies)))
        T = max(1, min(int(_log(rng, 1, 32_768)), int(MOST_FLOPS / 2 / n / k / W)))
        case = dict(what=what, W=W, E=E, T=T, n=n, k=k, type=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    offsets=rng.choice(["i32", "i64"]), empty=rng.choice([0.0, 0.1, 0.5]), pad=rng.random() < 0.3)
        if what == "product":
            return dict(case, back=rng.random() < 0.5, out=rng.choice(list(TYPES)))
        return dict(case, accumulate=rng.random() < 0.3,
                    lead=rng.choice([0, 0, 4 * rng.randint(1, 5_000), rng.randint(1, 5_000)]))
    groups = rng.choice([1, 1, rng.randint(2, 16)])
    most = int(_log(rng, 64, 2e7))
    # sizes are spread over their logarithm: their mean is some most / log(most)
    count = max(1, min(int(_log(rng, 1, 1_000)), int(MOST_ELEMENTS / groups / most * math.log(most))))
    return dict(what=what, tensors="random", count=count, most=most, groups=groups, type=rng.choice(list(TYPES)),
                shapes=rng.randrange(1 << 30), gap=rng.choice([0, 0, rng.randint(1, 100)]),
                packed=rng.random() < 0.5)


# ------------------------------------------------------------ tensors' shapes

def _conv_shapes():
    """Convolutions and normalisations of a 50-layer bottleneck image model, as matrices and vectors."""
    shapes, width = [(64, 147), (1, 64), (1, 64)], 64
    for blocks, mid in ((3, 64), (4, 128), (6, 256), (3, 512)):
        for b in range(blocks):
            shapes += [(mid, width), (1, mid), (1, mid), (mid, 9 * mid), (1, mid), (1, mid), (4 * mid, mid),
                       (1, 4 * mid), (1, 4 * mid)]
            if b == 0:
                shapes += [(4 * mid, width), (1, 4 * mid), (1, 4 * mid)]
            width = 4 * mid
    return shapes + [(1_000, 2_048), (1, 1_000)]


def _decoder_shapes():
    """24 blocks of width 2048, their table of 50,257 tokens and its 2,048 positions."""
    d = 2_048
    block = [(1, d), (1, d), (3 * d, d), (1, 3 * d), (d, d), (1, d), (1, d), (1, d), (4 * d, d), (1, 4 * d), (d, 4 * d),
             (1, d)]
    return [(50_257, d), (2_048, d)] + 24 * block + [(1, d), (1, d)]


def _shapes(case):
    """The tensors of one group."""
    if case["tensors"] == "conv":
        return _conv_shapes()
    if case["tensors"] == "decoder":
        return _decoder_shapes()
    rng = random.Random(case["shapes"])
    shapes = []
    for _ in range(case["count"]):
        n = int(_log(rng, 1, case["most"] + 0.9))
        rows = int(_log(rng, 1, n + 0.9)) if n > 1 and rng.random() < 0.6 else 1
        shapes.append((rows, n // rows))
    return shapes


def work(case):
    size = lambda t: TYPES[t].itemsize  # noqa: E731
    if case["what"] in ("product", "grad"):
        W, T, E, n, k = (case[i] for i in ("W", "T", "E", "n", "k"))
        T = W * (T - T // 8 if case["pad"] else T)
        flops = 2 * T * n * k
        if case["what"] == "grad":
            moved = (8 if case["accumulate"] else 4) * W * E * n * k
            return {"bytes": T * (n + k) * size(case["type"]) + moved, "flops": flops}
        read, written = (n, k) if case["back"] else (k, n)
        used = max(1, round(min(E * (1 - case["empty"]), T)))  # a matrix without a token need not be read
        return {"bytes": (T * read + used * n * k) * size(case["type"]) + T * written * size(case["out"]),
                "flops": flops}
    elements = case["groups"] * sum(r * c for r, c in _shapes(case))
    moved = size(case["type"]) + (4 if case["what"] == "clip" else 0)
    return {"bytes": elements * moved, "flops": elements * (3 if case["what"] == "clip" else 2)}


# -------------------------------------------------------------------- inputs

def _sizes(g, case):
    """How many rows each worker's experts have."""
    T, E = case["T"], case["E"]
    T = T - T // 8 if case["pad"] else T
    sizes = []
    for _ in range(case["W"]):
        p = torch.exp(0.7 * torch.randn(E, generator=g))
        gone = torch.rand(E, generator=g) < case["empty"]
        if not bool(gone.all()):
            p[gone] = 0.0
        sizes.append(torch.bincount(torch.multinomial(p, T, replacement=True, generator=g), minlength=E).tolist())
    return sizes


def _tokens(case, s):
    g = torch.Generator(device=DEV).manual_seed(s["seed"])
    host = torch.Generator().manual_seed(s["seed"])
    W, T, E, n, k = (case[i] for i in ("W", "T", "E", "n", "k"))
    s["sizes"] = _sizes(host, case)
    off = torch.tensor(s["sizes"], dtype=torch.int64).cumsum(1)
    off = torch.cat([torch.zeros(W, 1, dtype=torch.int64), off], 1)
    s["offsets"] = off.to(torch.int32 if case["offsets"] == "i32" else torch.int64).to(DEV)
    kind = TYPES[case["type"]]
    rand = lambda scale, *size: (torch.randn(*size, generator=g, device=DEV) * scale).to(kind)  # noqa: E731
    if case["what"] == "product":
        s["w"] = rand(k ** -0.5, E, n, k)
        s["x"] = rand(1e-3, W, T, n) if case["back"] else rand(1.0, W, T, k)
        s["y"] = torch.zeros(W, T, k if case["back"] else n, dtype=TYPES[case["out"]], device=DEV)
        return s
    s["dy"], s["x"] = rand(1e-3, W, T, n), rand(1.0, W, T, k)
    stride = (case["lead"] + E * n * k + 63) // 64 * 64
    # the workers' rows; what is accumulated onto is the gradient of the micro-batch before
    s["rows"] = torch.randn(W, stride, generator=g, device=DEV) * 1e-2 if case["accumulate"] else \
        torch.empty(W, stride, device=DEV)
    s["segment"] = s["rows"][:, case["lead"]:case["lead"] + E * n * k].unflatten(1, (E, n, k))
    return s


def prepare(case, seed):
    s = dict(case, seed=seed)
    if case["what"] in ("product", "grad"):
        return _tokens(case, s)
    g = torch.Generator(device=DEV).manual_seed(seed)
    G, shapes = case["groups"], _shapes(case)
    # where each tensor begins in its worker's memory: one after the other, or each allocated by itself
    at, places = 0, []
    for r, c in shapes:
        at = at if case["packed"] else (at + 127) // 128 * 128
        places.append(at)
        at += r * (c + case["gap"])
    flat = (torch.randn(G, at, generator=g, device=DEV) * 2e-3).to(TYPES[case["type"]])
    s["tensors"] = [[flat[w].as_strided((r, c), (c + case["gap"], 1), w * at + p) for (r, c), p in zip(shapes, places)]
                    for w in range(G)]
    s["norms"] = torch.empty(G, device=DEV)
    if case["what"] == "clip":
        total = sum(r * c for r, c in shapes)
        s["max_norm"] = 1e-3 * math.sqrt(total)  # half of what the norms are about
        s["rows"] = torch.empty(G, total, device=DEV)
        s["places"] = [[p.view(shape) for p, shape in zip(row.split([r * c for r, c in shapes]), shapes)]
                       for row in s["rows"]]
    return s


# ------------------------------------------------------------------ the pass

def run(state):
    return (_library if own else _plain)(state)


def _plan(nf, s):
    """The list of tensors, and the workspace, that a program keeps from step to step."""
    if "plan" not in s:
        tensors = [t for group in s["tensors"] for t in group]
        groups = [w for w, group in enumerate(s["tensors"]) for _ in group]
        places = [p for row in s["places"] for p in row] if "places" in s else None
        s["plan"] = nf.norm_plan(tensors, places, groups)
        s["ws"] = nf.empty_workspace(nf.nf_grad_norm_workspace_bytes(s["plan"]))
    return s["plan"], s["ws"]


def _library(s):
    import paper_2606_25759_amd as nf

    if s["what"] == "product":
        nf.nf_expert_product(s["x"], s["w"], s["offsets"], s["y"], transposed=s["back"])
        return s["y"]
    if s["what"] == "grad":
        if "ws" not in s:
            s["ws"] = nf.empty_workspace(nf.nf_expert_grad_workspace_bytes(s["W"], s["T"], s["E"], s["n"], s["k"]))
        nf.nf_expert_grad(s["dy"], s["x"], s["offsets"], s["rows"], s["lead"], s["ws"], accumulate=s["accumulate"])
        return s["segment"]
    plan, ws = _plan(nf, s)
    if s["what"] == "norm":
        nf.nf_grad_norm(plan, s["norms"], ws)
        return s["norms"]
    nf.nf_grad_norm_clip(plan, s["max_norm"], s["norms"], ws, eps=EPS)
    return s["norms"], s["rows"]


def _plain(s):
    if s["what"] == "product":
        x, w = s["x"].float(), s["w"].float()
        w = w if s["back"] else w.transpose(1, 2)
        for worker, sizes in enumerate(s["sizes"]):
            used = sum(sizes)
            parts = [rows @ w[e] for e, rows in enumerate(x[worker, :used].split(sizes)) if rows.shape[0]]
            s["y"][worker, :used] = torch.cat(parts).to(s["y"].dtype)
        return s["y"]
    if s["what"] == "grad":
        dy, x = s["dy"].float(), s["x"].float()
        for worker, sizes in enumerate(s["sizes"]):
            used = sum(sizes)
            parts = zip(dy[worker, :used].split(sizes), x[worker, :used].split(sizes), s["segment"][worker])
            for a, b, to in parts:
                if s["accumulate"]:
                    to.addmm_(a.t(), b)
                else:
                    torch.mm(a.t(), b, out=to)
        return s["segment"]
    for w, group in enumerate(s["tensors"]):
        s["norms"][w] = torch.stack([t.double().square().sum() for t in group]).sum().sqrt()
    if s["what"] == "norm":
        return s["norms"]
    coef = (s["max_norm"] / (s["norms"].double() + EPS)).clamp(max=1.0).float()
    for w, group in enumerate(s["tensors"]):
        for t, to in zip(group, s["places"][w]):
            torch.mul(t.float(), coef[w], out=to)
    return s["norms"], s["rows"]


# ------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["what"] == "product":
        out = s["y"].double()
        for w in range(case["W"]):
            ends = s["offsets"][w].tolist()
            for e in range(case["E"]):
                a, b = ends[e], ends[e + 1]
                m = s["w"][e].double()
                out[w, a:b] = s["x"][w, a:b].double() @ (m if case["back"] else m.t())
        return out
    if case["what"] == "grad":
        out = s["segment"].double() if case["accumulate"] else torch.zeros_like(s["segment"], dtype=torch.float64)
        for w in range(case["W"]):
            ends = s["offsets"][w].tolist()
            for e in range(case["E"]):
                a, b = ends[e], ends[e + 1]
                out[w, e] += s["dy"][w, a:b].double().t() @ s["x"][w, a:b].double()
        return out
    each = [[float(torch.linalg.vector_norm(t.double())) for t in group] for group in s["tensors"]]
    norms = [math.hypot(*group) for group in each]
    if case["what"] == "norm":
        return torch.tensor(norms, dtype=torch.float64, device=DEV)
    out = torch.empty(s["rows"].shape, dtype=torch.float64, device=DEV)
    for w, group in enumerate(s["tensors"]):
        ratio = min(1.0, s["max_norm"] / (norms[w] + EPS))
        at = 0
        for t in group:
            out[w, at:at + t.numel()] = t.double().reshape(-1) * ratio
            at += t.numel()
    return torch.tensor(norms, dtype=torch.float64, device=DEV), out
