"""SparseLoCo on a language model of one block, end to end on one GPU: R simulated workers train it on a synthetic text, H inner steps each, and
meet in the outer step.

    python -m paper_2508_15706_amd.block_example [--workers 2] [--rounds 4] [--inner-steps 10]

One inner step: the tokens' embeddings are normalised straight into 4-bit operands, multiplied to queries, keys and values, attended
(packed documents, grouped heads), multiplied, added to the residual and normalised into 4-bit operands again, and multiplied to logits;
the loss leaves its gradient in the logits' place; back through all of it; the gradients' norm; AdamW with 8-bit moments.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as sl
from .inner_example import Mx4Linear
from .synth import LAYOUT_FLAT, LAYOUT_TILE64


class BlockModel:
    """Parameters in one arena, and the buffers of a step over `tokens` tokens in documents that begin at `starts`."""

    def __init__(self, vocab: int, d: int, heads: int, kv_heads: int, dim: int, lengths, seed: int = 0):
        self.vocab, self.d, self.heads, self.kv_heads, self.dim = vocab, d, heads, kv_heads, dim
        self.tokens = n = sum(lengths)
        wide = (heads + 2 * kv_heads) * dim
        shapes = {"embed": (vocab, d), "qkv": (wide, d), "out": (d, heads * dim), "head": (vocab, d), "norm1": (1, d), "norm2": (1, d)}
        self.descs, self.part, off = [], {}, 0
        for name, (r, c) in shapes.items():
            self.descs.append((r, c, off, LAYOUT_TILE64 if r > 1 else LAYOUT_FLAT))
            self.part[name] = slice(off, off + r * c), (r, c) if r > 1 else (c,)
            off += -(-r * c // 256) * 256
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.theta = torch.zeros(off, device="cuda")
        for name, (r, c) in shapes.items():
            self.view(self.theta, name).normal_(0.0, 0.02 if name == "embed" else c ** -0.5, generator=g) if r > 1 else self.view(self.theta, name).fill_(1.0)
        self.theta16, self.grad = self.theta.bfloat16(), torch.zeros(off, device="cuda")
        self.opt = sl.sl_adamw_create(self.descs, [1.0 if r > 1 else 0.0 for r, _, _, _ in self.descs])
        self.m, self.v = (torch.zeros(off, dtype=torch.uint8, device="cuda") for _ in range(2))
        self.m_scales, self.v_scales = (torch.zeros(self.opt.num_blocks, dtype=torch.uint8, device="cuda") for _ in range(2))
        self.norm, self.norm_ws = torch.empty(2, device="cuda"), sl.alloc_norm_workspace(self.opt)
        self.layers = {"qkv": Mx4Linear(n, wide, d), "out": Mx4Linear(n, d, heads * dim), "head": Mx4Linear(n, vocab, d)}
        ends = [0]
        for length in lengths:
            ends.append(ends[-1] + length)
        self.starts = torch.tensor(ends, dtype=torch.int32, device="cuda")

        def f32(*s):
            return torch.empty(*s, device="cuda")

        def b16(*s):
            return torch.empty(*s, dtype=torch.bfloat16, device="cuda")
        self.h0, self.h1, self.rstd1, self.rstd2 = f32(n, d), f32(n, d), f32(n), f32(n)
        self.qkv, self.dqkv = b16(n, heads + 2 * kv_heads, dim), b16(n, heads + 2 * kv_heads, dim)
        self.mixed, self.lse, self.added = b16(n, heads, dim), f32(heads, n), b16(n, d)
        self.logits, self.loss, self.logp = b16(n, vocab), f32(1), f32(n)
        self.dh = f32(n, d)
        self.attend_ws, self.loss_ws = sl.alloc_attention_workspace(n, heads, kv_heads=kv_heads, dim=dim), sl.alloc_token_loss_workspace(n)
        self.rms_ws = sl.alloc_rms_norm_workspace(n, d)
        self.error = torch.zeros(off, device="cuda")
        self.step = 0

    def view(self, arena: torch.Tensor, name: str) -> torch.Tensor:
        where, shape = self.part[name]
        return arena[where].view(shape)

    def parts(self, t: torch.Tensor):
        """Queries, keys and values of (tokens, heads + 2 kv_heads, dim): views."""
        h, k = self.heads, self.kv_heads
        return t[:, :h], t[:, h:h + k], t[:, h + k:]

    def forward(self, tokens: torch.Tensor, targets: torch.Tensor, weights: torch.Tensor) -> None:
        """Leaves the loss, and its gradient in the logits' place."""
        L = self.layers
        for name, layer in L.items():
            layer.set_weight(self.view(self.theta16, name))
        torch.index_select(self.view(self.theta, "embed"), 0, tokens, out=self.h0)
        sl.sl_rms_norm(self.h0, self.view(self.theta, "norm1"), None, rstd=self.rstd1, q=L["qkv"].x, qt=L["qkv"].xt)
        sl.sl_mx4_product(L["qkv"].x, L["qkv"].w, self.qkv.view(self.tokens, -1), self.d, L["qkv"].ws)
        q, k, v = self.parts(self.qkv)
        sl.sl_attention(q, k, v, self.mixed, self.starts, lse=self.lse)
        sl.sl_mx4_quantize(self.mixed.view(self.tokens, -1), L["out"].x, L["out"].xt)
        sl.sl_mx4_product(L["out"].x, L["out"].w, self.added, self.heads * self.dim, L["out"].ws)
        sl.sl_rms_norm(self.added, self.view(self.theta, "norm2"), None, residual=self.h0, h=self.h1, rstd=self.rstd2, q=L["head"].x, qt=L["head"].xt)
        sl.sl_mx4_product(L["head"].x, L["head"].w, self.logits, self.d, L["head"].ws)
        sl.sl_token_loss(self.logits, targets, weights, self.loss, logp=self.logp, dlogits=self.logits, workspace=self.loss_ws)

    def backward_to_embeddings(self) -> None:
        """Gradients of the layers' parameters, and of the tokens' embeddings in dh, from what forward left: nothing that sorts, so that a graph may hold it."""
        L, g = self.layers, self.grad
        self.dy2 = L["head"].backward(self.logits, self.view(g, "head"))
        sl.sl_rms_norm_backward(self.h1, self.view(self.theta, "norm2"), self.rstd2, self.dy2, self.dh, dw=self.view(g, "norm2"), workspace=self.rms_ws)
        self.dmixed = L["out"].backward(self.dh.bfloat16(), self.view(g, "out")).view(self.tokens, self.heads, self.dim)
        q, k, v = self.parts(self.qkv)
        dq, dk, dv = self.parts(self.dqkv)
        sl.sl_attention_backward(q, k, v, self.mixed, self.lse, self.dmixed, dq, dk, dv, self.starts, workspace=self.attend_ws)
        self.dy1 = L["qkv"].backward(self.dqkv.view(self.tokens, -1), self.view(g, "qkv"))
        sl.sl_rms_norm_backward(self.h0, self.view(self.theta, "norm1"), self.rstd1, self.dy1, self.dh, dh=self.dh, dw=self.view(g, "norm1"), workspace=self.rms_ws)

    def embedding_gradient(self, tokens: torch.Tensor) -> None:
        embed = self.view(self.grad, "embed")
        embed.zero_()
        embed.index_put_((tokens,), self.dh, accumulate=True)

    def backward(self, tokens: torch.Tensor) -> None:
        """Gradients of all parameters from what forward left."""
        self.backward_to_embeddings()
        self.embedding_gradient(tokens)

    def update(self, lr: float, seed: int) -> None:
        sl.sl_grad_norm(self.opt, self.grad, 1.0, self.norm, self.norm_ws)
        self.step += 1
        sl.sl_adamw_step8(self.opt, self.theta, self.grad, self.m, self.v, self.m_scales, self.v_scales, seed=seed * 1000003 + self.step, lr=lr,
                          beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=self.step, grad_scale=self.norm[1:], theta16=self.theta16)

    def load(self, theta: torch.Tensor) -> None:
        self.theta.copy_(theta)
        self.theta16.copy_(theta)


def text(model: BlockModel, g: torch.Generator):
    """Documents of a chain in which a token names the next one, nine times in ten; the last token of a document has no target."""
    n, vocab = model.tokens, model.vocab
    tokens = torch.randint(vocab, (n,), device="cuda", generator=g)
    keep = torch.rand(n, device="cuda", generator=g) < 0.9
    for i in range(1, n):
        tokens[i] = torch.where(keep[i], (tokens[i - 1] * 5 + 3) % vocab, tokens[i])
    targets = torch.roll(tokens, -1)
    targets[(model.starts[1:] - 1).long()] = -1
    return tokens, targets


def train(workers: int = 2, rounds: int = 4, inner_steps: int = 10, vocab: int = 500, d: int = 128, heads: int = 4, kv_heads: int = 2, dim: int = 32,
          lengths=(100, 37, 1, 120), k: int = 64, lr: float = 3e-3, beta: float = 0.95, outer_lr: float = 1.0, seed: int = 0):
    """-> losses, one per round: the mean over the round's inner steps and workers."""
    team = [BlockModel(vocab, d, heads, kv_heads, dim, lengths, seed) for _ in range(workers)]
    theta = team[0].theta.clone()
    plan = sl.sl_plan_create(team[0].descs, k)
    ws = sl.alloc_workspace(plan)
    payloads = [sl.alloc_payload(plan) for _ in team]
    data = [torch.Generator(device="cuda").manual_seed(seed + 1 + r) for r in range(workers)]
    batches = [[text(m, g) for _ in range(2)] for m, g in zip(team, data)]
    weights = torch.full((team[0].tokens,), 1.0 / team[0].tokens, device="cuda")
    losses = []
    for _ in range(rounds):
        total = torch.zeros((), device="cuda")
        for r, (model, payload) in enumerate(zip(team, payloads)):
            model.load(theta)
            for i in range(inner_steps):
                tokens, targets = batches[r][i % 2]
                model.forward(tokens, targets, weights)
                model.backward(tokens)
                model.update(lr, seed + r)
                total += model.loss[0]
            sl.sl_compress_params(plan, model.error, theta, model.theta, beta, payload, ws)
        sl.sl_decompress_avg_apply(plan, theta, payloads, outer_lr)
        losses.append(total / (workers * inner_steps))
    team[0].load(theta)
    return [float(x) for x in losses], team[0]


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workers", type=int, default=2)
    ap.add_argument("--rounds", type=int, default=4)
    ap.add_argument("--inner-steps", type=int, default=10)
    a = ap.parse_args()
    for i, loss in enumerate(train(a.workers, a.rounds, a.inner_steps)[0]):
        print(f"round {i + 1}: mean loss of its inner steps {loss:.4f}")


if __name__ == "__main__":
    main()
