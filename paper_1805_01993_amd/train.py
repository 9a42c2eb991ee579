"""A training loop on an emulated cluster: the Map phase is the gradient of a trained block, file by file, and the coded
shuffle sums it.

    python -m paper_1805_01993_amd.train [--nodes 8] [--replication 2] [--width 256] [--hidden 512] [--tokens 64]
                                         [--steps 20] [--mode bf16] [--dropout 0.1]

The block predicts targets from its inputs: n = norm(x), f = feed-forward(n), y = scale x + gate D(norm(f)), loss
|y - target|^2 / 2 per element.  A step

  maps       every file to the gradient of its own tokens: a join, the feed-forward block, a join, and back (ccdc_join_*,
             ccdc_ffn_*); the gradients of one file are its row of V, [W_in | W_out | w_pre | w_post | gate]
  shuffles   ccdc_pipeline_fused: coded packets, and in Phi every parameter's gradient summed over the files
  updates    the parameters on their reducers

Node k of a cluster would map only the files it stores.  What it makes of them is the same bits that every other node storing
them has (`own_rows`), dropout included: the masks are drawn from the file's number, not from a node's state.  That is what
lets a receiver cancel the packets that it knows.
"""
from __future__ import annotations

import argparse
import math

import torch

from .binding import ccdc_block, ccdc_plan

TORCH = {"f32": torch.float32, "h32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


class Trainer:
    """The cluster's plan, the block and its parameters (fp32 masters), and a data set of one token matrix a file."""

    def __init__(self, nodes, replication, width, hidden, tokens, mode="bf16", dropout=0.1, seed=0, residual_scale=0.5):
        self.width, self.hidden, self.mode, self.dropout, self.scale = width, hidden, mode, dropout, residual_scale
        files = math.comb(nodes, replication)
        self.tokens = [tokens] * files if isinstance(tokens, int) else list(tokens)
        self.sizes = {"W_in": (2 * hidden, width), "W_out": (width, hidden), "w_pre": (width,), "w_post": (width,), "gate": (width,)}
        count = sum(math.prod(s) for s in self.sizes.values())
        T = -(-count // nodes)                               # the row of a file, cut into one value per node
        T = -(-T // 8) * 8
        self.plan = ccdc_plan(nodes, replication, nodes, files).bind(T, mode).upload()
        shapes, dtype = self.plan.shapes(), TORCH[mode]
        g = torch.Generator().manual_seed(seed)
        start = {"W_in": torch.randn(self.sizes["W_in"], generator=g) / math.sqrt(width),
                 "W_out": torch.randn(self.sizes["W_out"], generator=g) / math.sqrt(hidden),
                 "w_pre": torch.ones(width), "w_post": torch.ones(width), "gate": torch.full((width,), 0.1)}
        self.master = torch.zeros(nodes * T, device="cuda")
        self.master[:count] = torch.cat([start[k].reshape(-1) for k in self.sizes]).cuda()
        rows = sum(self.tokens)
        self.x = torch.randn(rows, width, generator=g).to(dtype).cuda()
        self.target = (self.x.float() * residual_scale + torch.randn(width, generator=g).cuda() * torch.tanh(self.x.float())).to(dtype)
        self.V = torch.zeros(shapes["V"], dtype=dtype, device="cuda")        # what a row has past the parameters stays zero
        self.X = torch.empty(shapes["X"], dtype=dtype, device="cuda")
        self.Phi = torch.empty(shapes["Phi"], dtype=dtype, device="cuda")
        self.every = self._batch(range(files))

    def _batch(self, files):
        """The block bound to these files, and the buffers of a step on them."""
        files = list(files)
        block = ccdc_block(self.width, self.hidden, self.mode, residual_scale=self.scale, dropout_hidden=self.dropout,
                           dropout_out=self.dropout).bind([self.tokens[n] for n in files], files).upload()
        # the norm of x alone, in front: a join scales what it norms, so this one's scale is one
        first = ccdc_block(self.width, 1, self.mode).bind([self.tokens[n] for n in files], files).upload()
        rows = block.tokens
        new = lambda: torch.empty(rows, self.width, dtype=self.x.dtype, device="cuda")  # noqa: E731
        return {"block": block, "first": first, "saved": torch.empty(block.saved_bytes, dtype=torch.uint8, device="cuda"),
                "n": new(), "f": new(), "y": new(), "df": new(), "dn": new()}

    def parameters(self):
        """The parameters as the step's products take them."""
        flat, at, out = self.master.to(self.x.dtype), 0, {}
        for name, shape in self.sizes.items():
            out[name] = flat[at:at + math.prod(shape)].view(shape)
            at += math.prod(shape)
        return out

    def map(self, batch, x, target, V, seed):
        """V[n] = gradient of file n's loss; returns the loss over the batch."""
        p, block, s = self.parameters(), batch["block"], batch
        rows, at, grad = V.view(V.shape[-3], -1), 0, {}
        for name, shape in self.sizes.items():
            grad[name] = rows[:, at:at + math.prod(shape)].unflatten(1, shape)
            at += math.prod(shape)
        s["first"].join_forward(x, None, None, s["n"], w_pre=p["w_pre"])
        block.ffn_forward(s["n"], p["W_in"], p["W_out"], s["f"], saved=s["saved"], seed=seed)
        block.join_forward(x, s["f"], s["y"], None, w_post=p["w_post"], gate=p["gate"], seed=seed)
        off = s["y"].float() - target.float()
        block.join_backward(None, off.to(x.dtype), None, s["f"], None, s["df"], w_post=p["w_post"], gate=p["gate"],
                            dw_post=grad["w_post"], dgate=grad["gate"], seed=seed)
        block.ffn_backward(s["n"], p["W_in"], p["W_out"], s["saved"], s["df"], s["dn"], grad["W_in"], grad["W_out"])
        s["first"].join_backward(s["dn"], None, x, None, None, None, w_pre=p["w_pre"], dw_pre=grad["w_pre"])
        return off.square().mean() / 2

    def step(self, number, rate=0.5):
        """One training step; returns its loss (a tensor on the device)."""
        loss = self.map(self.every, self.x, self.target, self.V, seed=number)
        self.plan.pipeline_fused(self.V, self.X, self.Phi)
        self.master -= rate / self.x.shape[0] * self.Phi.view(-1).float()
        return loss

    def own_rows(self, node, number):
        """What node `node` maps in step `number`: the numbers of its files, and their rows of V."""
        files = [int(n) for n in self.plan.node_files()[node]]
        ends = torch.tensor(self.tokens).cumsum(0).tolist()
        rows = torch.cat([torch.arange(ends[n] - self.tokens[n], ends[n]) for n in files]).cuda()
        V = torch.zeros((len(files),) + tuple(self.V.shape[2:]), dtype=self.V.dtype, device="cuda")
        self.map(self._batch(files), self.x[rows], self.target[rows], V, seed=number)
        return files, V


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, default in (("nodes", 8), ("replication", 2), ("width", 256), ("hidden", 512), ("tokens", 64), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--mode", choices=sorted(TORCH), default="bf16")
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--rate", type=float, default=0.5)
    a = ap.parse_args(argv)
    t = Trainer(a.nodes, a.replication, a.width, a.hidden, a.tokens, a.mode, a.dropout)
    print(f"{a.nodes} nodes, {len(t.tokens)} files on {a.replication} of them each, {t.x.shape[0]} tokens, "
          f"{t.plan.Q * t.plan.T} parameters a row, {a.mode}")
    for number in range(a.steps):
        loss = t.step(number, a.rate)
        if number % max(1, a.steps // 10) == 0 or number == a.steps - 1:
            print(f"step {number}: loss {float(loss):.4f}", flush=True)
    files, V = t.own_rows(0, a.steps)
    t.map(t.every, t.x, t.target, t.V, seed=a.steps)
    same = torch.equal(V, t.V[0, files])
    print(f"node 0 maps its {len(files)} files to the same bits: {same}")
    return 0 if same else 1


if __name__ == "__main__":
    raise SystemExit(main())
