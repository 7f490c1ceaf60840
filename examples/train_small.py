"""A small model trained by W simulated workers on one GPU, every part of the step that the library has:

    lookup -> forward and backward (torch) -> the table's gradient into the worker's row
           -> the bucket reducer over all rows -> orthogonalised update of the matrices

The model predicts the next token of a random first-order chain: embedding table [V, d], a hidden layer of h units
between two matrices, a head [V, d].  All parameters lie in one flat buffer; the two matrices are low-bit eligible,
the table and the head are FP32-routed, as the reducer's bindings have it.

    python examples/train_small.py --steps 60 --format ternary
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_25759_amd as nf  # noqa: E402


class Trainer:
    def __init__(self, W=4, T=512, V=1000, d=128, h=256, lr=0.02, format=nf.NF_FORMAT_BINARY, seed=0):
        self.W, self.T, self.V, self.d, self.h, self.lr = W, T, V, d, h, lr
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        sizes = [("table", (V, d), 0), ("up", (h, d), 1), ("down", (d, h), 1), ("head", (V, d), 0)]
        self.at, n = {}, 0
        for name, shape, _ in sizes:
            self.at[name] = (n, shape)
            n += shape[0] * shape[1]
        self.n = n
        dev = "cuda"
        self.theta = torch.empty(n, device=dev)
        for name, shape, _ in sizes:
            self.view(self.theta, name).normal_(0.0, 1.0 / shape[1] ** 0.5, generator=self.gen)
        self.momentum = torch.zeros(n, device=dev)
        self.rows = torch.zeros(W, (n + 3) // 4 * 4, device=dev)  # the workers' gradients
        # the reducer's buffers
        self.bucket_n = (n // 3 + 63) // 64 * 64
        nb = -(-n // self.bucket_n)
        mask = nf.nf_mask_from_segments([self.at[k][0] for k, _, _ in sizes],
                                        [s[0] * s[1] for _, s, _ in sizes], [e for _, _, e in sizes], n)
        self.mask = torch.from_numpy(mask.view(np.int64)).to(dev)
        self.policy = nf.policy(fp32_op=nf.NF_FP32_MEAN, format=format)
        planes = 2 if format == nf.NF_FORMAT_TERNARY else 1
        self.bits = torch.empty(planes * W, (n + 63) // 64, dtype=torch.int64, device=dev)
        self.out = torch.empty(n, device=dev)
        self.stats = torch.empty(nb * W * nf.STATS_BYTES, dtype=torch.uint8, device=dev)
        self.decisions = torch.empty(nb * nf.DECISION_BYTES, dtype=torch.uint8, device=dev)
        self.reduce_ws = nf.empty_workspace(nf.nf_workspace_bytes_buckets(W, n, self.bucket_n))
        self.nb = nb
        # the operators': made once, kept from step to step
        self.scale = d ** 0.5
        self.emb_ws = nf.empty_workspace(nf.nf_embedding_workspace_bytes(W, T, V, d))
        self.how = nf.orthogonal()
        self.matrix_ws = nf.empty_workspace(max(nf.nf_orthogonal_workspace_bytes(*self.at[k][1], 1, self.how)
                                                for k in ("up", "down")))
        # the chain: every token has a few likely successors
        self.successors = torch.randint(0, V, (V, 4), generator=self.gen, device=dev)

    def view(self, flat, name):
        at, (r, c) = self.at[name]
        return flat[at:at + r * c].view(r, c)

    def batch(self):
        W, T = self.W, self.T
        ids = torch.randint(0, self.V, (W, T), generator=self.gen, device="cuda")
        pick = torch.randint(0, 4, (W, T), generator=self.gen, device="cuda")
        return ids, self.successors[ids, pick]

    def step(self):
        ids, targets = self.batch()
        W, T, d = self.W, self.T, self.d
        x = torch.empty(W, T, d, device="cuda")
        nf.nf_embedding_lookup(self.view(self.theta, "table"), ids.view(-1), x.view(W * T, d), scale=self.scale)
        x.requires_grad_(True)
        dy, loss = torch.empty(W, T, d, device="cuda"), 0.0
        for w in range(W):  # each worker's forward and backward, its matrices' gradients into its row
            p = {k: self.view(self.theta, k).detach().requires_grad_(True) for k in ("up", "down", "head")}
            y = x[w] + torch.relu(x[w] @ p["up"].t()) @ p["down"].t()
            part = torch.nn.functional.cross_entropy(y @ p["head"].t(), targets[w])
            grads = torch.autograd.grad(part, [x, *p.values()])
            dy[w] = grads[0][w]
            for k, g in zip(p, grads[1:]):
                self.view(self.rows[w], k).copy_(g)
            loss += part.detach() / W
        nf.nf_embedding_grad(dy, ids, self.rows, self.at["table"][0], self.V, self.emb_ws, scale=self.scale)
        nf.nf_route_buckets(self.rows, self.n, self.bucket_n, self.mask, self.policy, self.bits, None, self.out,
                            self.stats, self.decisions, self.reduce_ws)
        for k in ("up", "down"):
            r, c = self.at[k][1]
            step = nf.matrix_step(lr=self.lr, momentum=0.9, scale=0.2 * max(r, c) ** 0.5)
            nf.nf_orthogonal_update(self.view(self.out, k), self.view(self.momentum, k), self.view(self.theta, k), step,
                                    self.how, self.matrix_ws)
        for k in ("table", "head"):  # what is FP32-routed: plain momentum
            m = self.view(self.momentum, k).mul_(0.9).add_(self.view(self.out, k))
            self.view(self.theta, k).sub_(m, alpha=20 * self.lr)
        return float(loss)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--format", choices=("binary", "ternary"), default="binary")
    a = ap.parse_args(argv)
    t = Trainer(W=a.workers, format=nf.NF_FORMAT_TERNARY if a.format == "ternary" else nf.NF_FORMAT_BINARY)
    losses = []
    for k in range(a.steps):
        losses.append(t.step())
        if k % 10 == 0 or k == a.steps - 1:
            routes = nf.decisions_host(t.decisions, t.nb)["route"]
            print(f"step {k:4d}  loss {losses[-1]:.4f}  routes {''.join('LFP'[r] for r in routes)}", flush=True)
    return losses


if __name__ == "__main__":
    main()
