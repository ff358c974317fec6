"""A small token model with a layer of experts, trained and then asked, on the library's operators.

    python examples/train_experts.py [--steps 200] [--type bf16]

x = table[token] (tc_embed); a router picks 2 of 8 experts (tc_route); the experts' clamped two-layer networks run on the rows that
they were given (tc_expert_mm); their weighted sum (tc_expert_sum) is added to x; logits are products with the table again.  The
task: the next token is a fixed function of the current one.  Gradients of all operators come from the library too; torch
does the loss, the two dense products and the optimizer.  Weights are kept in fp32 and cast for the products.  Afterwards the model
continues sequences token by token, with the same operators at a batch of a few rows.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1802_04730_amd import tc355 as tc  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _bytes(n, device):
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


class Embed(torch.autograd.Function):
    """scale * table[tokens]."""

    @staticmethod
    def forward(ctx, table, tokens, scale):
        out = table.new_empty((tokens.shape[0], table.shape[1]))
        tc.tc_embed(table, tokens, out, scale)
        ctx.save_for_backward(tokens)
        ctx.rows, ctx.scale = table.shape[0], scale
        return out

    @staticmethod
    def backward(ctx, grad):
        (tokens,) = ctx.saved_tensors
        (T, D), E = grad.shape, ctx.rows
        out = grad.new_empty((E, D))
        tc.tc_embed_grad(grad.contiguous(), tokens, out, _bytes(tc.tc_embed_grad_workspace_bytes(E, D, T), grad.device), ctx.scale)
        return out, None, None


class Route(torch.autograd.Function):
    """Weights of the k experts of each token, their numbers, and the rows in the experts' order."""

    @staticmethod
    def forward(ctx, logits, k):
        T, E = logits.shape
        ints = lambda *s: torch.empty(s, dtype=torch.int32, device=logits.device)  # noqa: E731
        weights, chosen, offsets, rows, places = torch.empty((T, k), device=logits.device), ints(T, k), ints(E + 1), ints(T * k), ints(T, k)
        tc.tc_route(logits, weights, chosen, offsets, rows, places, _bytes(tc.tc_route_workspace_bytes(T, E, k), logits.device), norm=True)
        ctx.save_for_backward(logits, chosen)
        ctx.mark_non_differentiable(chosen, offsets, rows, places)
        return weights, chosen, offsets, rows, places

    @staticmethod
    def backward(ctx, grad, *_):
        logits, chosen = ctx.saved_tensors
        out = torch.empty_like(logits)
        tc.tc_route_grad(logits, chosen, grad.contiguous(), out, norm=True)
        return out, None


class Experts(torch.autograd.Function):
    """sum_i w_i * W2[e_i] max(W1[e_i] x, 0) over the experts e_i of each token."""

    @staticmethod
    def forward(ctx, x, w1, w2, weights, offsets, rows, places):
        R = rows.shape[0]
        hidden, y, out = x.new_empty((R, w1.shape[1])), x.new_empty((R, w2.shape[1])), torch.empty_like(x)
        tc.tc_expert_mm(x, w1, offsets, rows, hidden, relu=True)
        tc.tc_expert_mm(hidden, w2, offsets, None, y)
        tc.tc_expert_sum(y, weights, places, out)
        ctx.save_for_backward(x, w1, w2, weights, offsets, rows, places, hidden, y)
        return out

    @staticmethod
    def backward(ctx, grad):
        x, w1, w2, weights, offsets, rows, places, hidden, y = ctx.saved_tensors
        (E, H, D), R = w1.shape, rows.shape[0]
        ws = _bytes(tc.tc_expert_mm_grad_w_workspace_bytes(R, E, H, D), x.device)
        dy, dweights, dhidden = torch.empty_like(y), torch.empty_like(weights), torch.empty_like(hidden)
        dw1, dw2, drows, dx = torch.empty_like(w1), torch.empty_like(w2), y.new_empty((R, D)), torch.empty_like(x)
        tc.tc_expert_sum_grad(grad.contiguous(), y, weights, places, dy, dweights)
        tc.tc_expert_mm_grad_w(dy, hidden, offsets, None, dw2, ws)
        tc.tc_expert_mm_grad_x(dy, w2, offsets, hidden, dhidden)  # (0 where the hidden unit was clamped)
        tc.tc_expert_mm_grad_w(dhidden, x, offsets, rows, dw1, ws)
        tc.tc_expert_mm_grad_x(dhidden, w1, offsets, None, drows)
        tc.tc_expert_sum(drows, None, places, dx)  # the rows of a token's experts, added up
        return dx, dw1, dw2, dweights, None, None, None


class Model(torch.nn.Module):
    def __init__(self, vocabulary, width, hidden, experts, chosen, dtype):
        super().__init__()
        p = lambda *s, std: torch.nn.Parameter(torch.randn(*s) * std)  # noqa: E731
        self.table, self.router = p(vocabulary, width, std=width ** -0.5), p(experts, width, std=width ** -0.5)
        self.w1, self.w2 = p(experts, hidden, width, std=width ** -0.5), p(experts, width, hidden, std=hidden ** -0.5)
        self.chosen, self.dtype = chosen, dtype

    def forward(self, tokens):
        table = self.table.to(self.dtype)
        x = Embed.apply(table, tokens, float(table.shape[1]) ** 0.5)
        weights, _, offsets, rows, places = Route.apply((x @ self.router.to(self.dtype).t()).contiguous(), self.chosen)
        x = x + Experts.apply(x, self.w1.to(self.dtype), self.w2.to(self.dtype), weights, offsets, rows, places)
        return x @ table.t()


def main(steps=200, kind="bf16", vocabulary=512, width=128, hidden=256, experts=8, chosen=2, batch=2048, quiet=False):
    """Loss of the first and the last step, and the share of right tokens when the model continues sequences."""
    torch.manual_seed(0)
    follows = torch.randperm(vocabulary, device="cuda")
    model = Model(vocabulary, width, hidden, experts, chosen, TYPES[kind]).cuda()
    optimizer = torch.optim.Adam(model.parameters(), lr=3e-3)
    losses = []
    for step in range(steps):
        tokens = torch.randint(0, vocabulary, (batch,), device="cuda", dtype=torch.int32)
        loss = torch.nn.functional.cross_entropy(model(tokens).float(), follows[tokens.long()])
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        if step in (0, steps - 1) or step % 50 == 0:
            losses.append(loss.item())
            if not quiet:
                print("step %4d  loss %.4f" % (step, losses[-1]), flush=True)
    with torch.no_grad():
        token, right, length = torch.arange(8, device="cuda", dtype=torch.int32), 0, 32
        for _ in range(length):
            following = model(token).float().argmax(dim=1)
            right += int((following == follows[token.long()]).sum())
            token = following.to(torch.int32)
    if not quiet:
        print("continuing 8 sequences for %d tokens: %d of %d right" % (length, right, 8 * length))
    return losses[0], losses[-1], right / (8 * length)


if __name__ == "__main__":
    a = argparse.ArgumentParser()
    a.add_argument("--steps", type=int, default=200)
    a.add_argument("--type", choices=sorted(TYPES), default="bf16")
    a = a.parse_args()
    main(a.steps, a.type)
