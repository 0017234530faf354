"""A feed-forward block whose tokens choose their experts, trained in bf16, and a shared projection with an adapter for each request in front of it.

    n = layer_norm(x);  logits = n router^T;  the top experts of each token and their weights
    y = x + sum over a token's experts of weight * expert(n)

Forward, tokens go into the order of their experts, through the experts' two layers (examples/expert_layers.py) and back; backward, the same way in
the other direction, with the gradients of the weights by the router's logits beside them.  Plain gradient descent moves weights in single precision.
Serving, every request's rows have a low-rank adapter of their own, or none, beside one projection that all share.

    python examples/routed_block.py [--steps 100]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2210_12415_amd as alt  # noqa: E402
from examples.expert_layers import Layer, buffer  # noqa: E402


class Norm:
    """Layer norm of bf16 rows with its gradients."""

    def __init__(self, handle, rows, width):
        self.h, self.d = handle, alt.norm_desc(rows, width)
        self.gamma, self.beta = torch.ones(width, device="cuda"), torch.zeros(width, device="cuda")
        self.dgamma, self.dbeta = torch.empty_like(self.gamma), torch.empty_like(self.beta)
        self.mean, self.rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        self.y, self.dx = (torch.empty(rows, width, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.ws = buffer(handle.layer_norm_grad_workspace_size(self.d))

    def forward(self, x):
        self.x = x
        self.h.layer_norm(self.d, x, self.y, gamma=self.gamma, beta=self.beta, mean=self.mean, rstd=self.rstd)
        return self.y

    def gradients(self, dy):
        self.h.layer_norm_grad(self.d, dy, self.x, self.mean, self.rstd, self.dx, gamma=self.gamma, dgamma=self.dgamma, dbeta=self.dbeta, **self.ws)
        return self.dx

    def update(self, rate):
        self.gamma.sub_(self.dgamma, alpha=rate)
        self.beta.sub_(self.dbeta, alpha=rate)


class RoutedBlock:
    def __init__(self, handle, tokens, width, hidden, experts, top_k, generator, bias=None):
        self.h, self.shape, self.bias = handle, (tokens, width, experts, top_k), bias
        rows = tokens * top_k
        self.norm = Norm(handle, tokens, width)
        self.router = Layer(handle, tokens, 1, width, experts, False, False, generator)
        self.up, self.down = Layer(handle, rows, experts, width, hidden, True, False, generator), Layer(handle, rows, experts, hidden, width, False, True, generator)
        self.all = torch.tensor([0, tokens], dtype=torch.int32, device="cuda")
        self.route_desc = alt.route_desc(tokens, experts, top_k, dtype=alt.BF16, renormalize=True)
        self.exchange = alt.exchange_desc(tokens, top_k, rows, width)
        self.experts, self.rows = (torch.empty(tokens, top_k, dtype=torch.int32, device="cuda") for _ in range(2))
        self.offsets = torch.empty(experts + 1, dtype=torch.int32, device="cuda")
        self.weights, self.dweights = (torch.empty(tokens, top_k, device="cuda") for _ in range(2))
        wide = lambda n: torch.zeros(n, width, dtype=torch.bfloat16, device="cuda")
        self.in_order, self.d_in_order, self.mixed, self.y, self.dn, self.dx = wide(rows), wide(rows), wide(tokens), wide(tokens), wide(tokens), wide(tokens)
        self.dlogits = torch.empty(tokens, experts, dtype=torch.bfloat16, device="cuda")
        self.route_ws = buffer(handle.route_workspace_size(self.route_desc))

    def add(self, a, b, out):
        self.h.eltwise_add(alt.BF16, out.numel(), a, b, out)
        return out

    def forward(self, x):
        n = self.norm.forward(x)
        self.logits = self.router.forward(n, self.all)
        self.h.route(self.route_desc, self.logits, self.experts, self.weights, self.rows, self.offsets, bias=self.bias, **self.route_ws)
        self.h.dispatch_rows(self.exchange, n, self.rows, self.in_order)
        self.answers = self.down.forward(self.up.forward(self.in_order, self.offsets), self.offsets)
        self.h.combine_rows(self.exchange, self.answers, self.rows, self.mixed, weights=self.weights)
        return self.add(x, self.mixed, self.y)

    def gradients(self, dy):
        """Gradients of everything from that of y; returns x's."""
        self.h.combine_rows_grad(self.exchange, dy, self.answers, self.rows, self.weights, self.d_in_order, self.dweights)
        self.down.by_weights(self.d_in_order)
        d_hidden = self.down.by_tokens(self.d_in_order)
        self.up.by_weights(d_hidden)
        self.h.combine_rows(self.exchange, self.up.by_tokens(d_hidden), self.rows, self.mixed)
        self.h.route_grad(self.route_desc, self.logits, self.experts, self.dweights, self.dlogits)
        self.router.by_weights(self.dlogits)
        dn = self.add(self.mixed, self.router.by_tokens(self.dlogits), self.dn)
        return self.add(dy, self.norm.gradients(dn), self.dx)

    def update(self, rate):
        for part in (self.norm, self.router, self.up, self.down):
            part.update(rate)

    def step(self, x, target, rate):
        """One step of gradient descent; returns the loss before it."""
        wrong = self.forward(x).float() - target
        self.gradients((2 * wrong / wrong.shape[1]).bfloat16())
        self.update(rate / x.shape[0])
        return float(wrong.square().mean())


class Served:
    """A projection that all requests share, and each request's adapter beside it."""

    def __init__(self, handle, width, outputs, adapters, rank, generator):
        make = lambda *shape, std: (torch.randn(*shape, generator=generator, device="cuda") * std).bfloat16()
        self.h, self.shape = handle, (outputs, width, adapters, rank)
        self.w, self.a, self.b = make(outputs, width, std=width ** -0.5), make(adapters, rank, width, std=width ** -0.5), make(adapters, outputs, rank, std=rank ** -0.5)
        self.scale = torch.full((adapters,), 0.5, device="cuda")

    def forward(self, x, adapter):
        outputs, width, adapters, rank = self.shape
        d = alt.adapters_desc(x.shape[0], outputs, width, adapters, rank)
        y = torch.empty(x.shape[0], outputs, dtype=torch.bfloat16, device="cuda")
        self.h.gemm_adapters(d, x, self.w, adapter, self.a, self.b, y, scale=self.scale, **buffer(self.h.gemm_adapters_workspace_size(d)))
        return y


def main(argv=None):
    p = argparse.ArgumentParser()
    p.add_argument("--steps", type=int, default=100)
    p.add_argument("--tokens", type=int, default=2000)
    p.add_argument("--width", type=int, default=256)
    p.add_argument("--hidden", type=int, default=512)
    p.add_argument("--experts", type=int, default=12)
    p.add_argument("--top", type=int, default=2)
    p.add_argument("--rate", type=float, default=0.5)
    a = p.parse_args(argv)
    generator, handle = torch.Generator(device="cuda").manual_seed(1), alt.Handle()
    x = torch.randn(a.tokens, a.width, generator=generator, device="cuda").bfloat16()
    teacher, block = (RoutedBlock(handle, a.tokens, a.width, a.hidden, a.experts, a.top, generator) for _ in range(2))
    target = teacher.forward(x).float()
    losses = [block.step(x, target, a.rate) for _ in range(a.steps)]
    counts = block.offsets.diff()
    served = Served(handle, a.width, a.width, 4, 8, generator)
    requests = torch.tensor([0] * 5 + [-1] * 3 + [2] * 7 + [3], dtype=torch.int32, device="cuda")
    together = served.forward(x[:16], requests)
    alone = torch.cat([served.forward(x[i:i + 1], requests[i:i + 1]) for i in range(16)])
    print("loss %.4f -> %.4f in %d steps; tokens of an expert %d to %d; 16 rows of five requests together and alone differ by %.3f %%"
          % (losses[0], losses[-1], a.steps, counts.min(), counts.max(), 100 * (together.float() - alone.float()).norm() / together.float().norm()))
    return losses


if __name__ == "__main__":
    main()
