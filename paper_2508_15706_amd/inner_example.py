"""SparseLoCo end to end on one GPU: R simulated workers train a two-layer network on a synthetic task, H inner steps
each, and meet in the outer step.

    python -m paper_2508_15706_amd.inner_example [--workers 4] [--rounds 6] [--inner-steps 15]

One inner step (a worker's own):  h = x W1^T, r = max(h, 0), y = r W2^T on 4-bit operands, both layers' gradients on
4-bit operands too; the norm of all gradients and its clipping factor; AdamW with 8-bit moments, which leaves the fp32
parameters and the bf16 copy that the next step quantises.  One outer step: the change of a worker's
parameters is compressed with error feedback, the payloads are averaged and applied.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as sl
from .synth import LAYOUT_TILE64


class Mx4Linear:
    """y = x W^T with W of (n, k), x, W and dy in 4 bits; buffers for batches of m rows are kept."""

    def __init__(self, m: int, n: int, k: int):
        self.m, self.n, self.k = m, n, k
        self.w, self.wt = sl.alloc_mx4(n, k), sl.alloc_mx4(k, n)
        self.x, self.xt = sl.alloc_mx4(m, k), sl.alloc_mx4(k, m)
        self.g, self.gt = sl.alloc_mx4(m, n), sl.alloc_mx4(n, m)
        size = max(sl.sl_mx4_workspace_bytes(*s) for s in ((m, n, k), (m, k, n), (n, k, m)))
        self.ws = torch.empty(max(16, size), dtype=torch.uint8, device="cuda")

    def set_weight(self, w: torch.Tensor) -> None:
        sl.sl_mx4_quantize(w, self.w, self.wt)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        sl.sl_mx4_quantize(x, self.x, self.xt)
        y = torch.empty(self.m, self.n, dtype=torch.bfloat16, device=x.device)
        sl.sl_mx4_product(self.x, self.w, y, self.k, self.ws)
        return y

    def backward(self, dy: torch.Tensor, dw: torch.Tensor, need_dx: bool = True):
        """dw: out, fp32, (n, k); -> dx"""
        sl.sl_mx4_quantize(dy, self.g, self.gt)
        sl.sl_mx4_product(self.gt, self.xt, dw, self.m, self.ws)
        if not need_dx:
            return None
        dx = torch.empty(self.m, self.k, dtype=torch.bfloat16, device=dy.device)
        sl.sl_mx4_product(self.g, self.wt, dx, self.n, self.ws)
        return dx

    def infer(self, x: torch.Tensor) -> torch.Tensor:
        """Any number of rows up to m, without what the backward pass needs."""
        y = torch.empty(x.shape[0], self.n, dtype=torch.bfloat16, device=x.device)
        sl.sl_mx4_linear(x, self.w, y, self.ws)
        return y


class Worker:
    """Parameters of W1 (hidden x d) and W2 (out x hidden) in one arena, and what belongs to them."""

    def __init__(self, d: int, hidden: int, out: int, batch: int, theta: torch.Tensor, seed: int):
        self.descs = [(hidden, d, 0, LAYOUT_TILE64), (out, hidden, hidden * d, LAYOUT_TILE64)]
        n = hidden * d + out * hidden
        self.theta = theta.clone()
        self.theta16 = self.theta.bfloat16()
        self.grad = torch.zeros(n, device="cuda")
        self.views = [(slice(off, off + r * c), (r, c)) for r, c, off, _ in self.descs]
        self.opt = sl.sl_adamw_create(self.descs)
        self.m, self.v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
        self.m_scales, self.v_scales = (torch.zeros(self.opt.num_blocks, dtype=torch.uint8, device="cuda") for _ in range(2))
        self.norm, self.norm_ws = torch.empty(2, device="cuda"), sl.alloc_norm_workspace(self.opt)
        self.layers = [Mx4Linear(batch, hidden, d), Mx4Linear(batch, out, hidden)]
        self.data = torch.Generator(device="cuda")
        self.data.manual_seed(seed)
        self.error = torch.zeros(n, device="cuda")
        self.step = 0
        self.seed = seed

    def load(self, theta: torch.Tensor) -> None:
        self.theta.copy_(theta)
        self.theta16.copy_(theta)

    def quantize_weights(self) -> None:
        for layer, (part, shape) in zip(self.layers, self.views):
            layer.set_weight(self.theta16[part].view(shape))

    def predict(self, x: torch.Tensor) -> torch.Tensor:
        return self.layers[1].infer(torch.relu(self.layers[0].infer(x)))

    def inner_step(self, x: torch.Tensor, target: torch.Tensor, lr: float) -> torch.Tensor:
        """One step on the mean squared error; -> the loss before it."""
        self.quantize_weights()
        h = self.layers[0].forward(x)
        r = torch.relu(h)
        y = self.layers[1].forward(r)
        diff = y.float() - target
        dy = (diff * (2.0 / diff.numel())).bfloat16()
        g1, g2 = (self.grad[part].view(shape) for part, shape in self.views)
        dr = self.layers[1].backward(dy, g2)
        self.layers[0].backward(dr * (h > 0), g1, need_dx=False)
        sl.sl_grad_norm(self.opt, self.grad, 1.0, self.norm, self.norm_ws)
        self.step += 1
        sl.sl_adamw_step8(self.opt, self.theta, self.grad, self.m, self.v, self.m_scales, self.v_scales,
                          seed=self.seed * 1000003 + self.step, lr=lr, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1,
                          step=self.step, grad_scale=self.norm[1:], theta16=self.theta16)
        return diff.square().mean()


def train(workers: int = 4, rounds: int = 6, inner_steps: int = 15, d: int = 256, hidden: int = 512, out: int = 64,
          batch: int = 512, k: int = 256, lr: float = 2e-3, beta: float = 0.95, outer_lr: float = 1.0, seed: int = 0):
    """-> losses, one per round: the mean over the round's inner steps and workers."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    teacher = torch.empty(out, d, device="cuda").normal_(0, d ** -0.5, generator=g)
    n = hidden * d + out * hidden
    theta = torch.empty(n, device="cuda").normal_(0, 0.05, generator=g)
    team = [Worker(d, hidden, out, batch, theta, seed + 1 + r) for r in range(workers)]
    plan = sl.sl_plan_create(team[0].descs, k)
    ws = sl.alloc_workspace(plan)
    payloads = [sl.alloc_payload(plan) for _ in team]
    losses = []
    for _ in range(rounds):
        total = torch.zeros((), device="cuda")
        for worker, payload in zip(team, payloads):
            worker.load(theta)
            for _ in range(inner_steps):
                x = torch.empty(batch, d, device="cuda").normal_(generator=worker.data)
                total += worker.inner_step(x.bfloat16(), torch.tanh(x @ teacher.t()), lr)
            sl.sl_compress_params(plan, worker.error, theta, worker.theta, beta, payload, ws)
        sl.sl_decompress_avg_apply(plan, theta, payloads, outer_lr)
        losses.append(total / (workers * inner_steps))
    team[0].load(theta)
    team[0].quantize_weights()
    return [float(x) for x in losses], team[0], teacher


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--rounds", type=int, default=6)
    ap.add_argument("--inner-steps", type=int, default=15)
    a = ap.parse_args()
    losses, model, teacher = train(a.workers, a.rounds, a.inner_steps)
    for i, loss in enumerate(losses):
        print(f"round {i + 1}: mean loss of its inner steps {loss:.4f}")
    x = torch.randn(1, teacher.shape[1], device="cuda")
    y = model.predict(x.bfloat16())
    print(f"one row through the averaged parameters: squared error {float((y.float() - torch.tanh(x @ teacher.t())).square().mean()):.4f}")


if __name__ == "__main__":
    main()
