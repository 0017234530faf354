"""A feed-forward block of experts, trained in bf16 and then served in 8 bits.

Tokens arrive sorted by their expert; each expert is two layers with a ReLU between them.  Training runs the block forward, takes the gradients
by the tokens, the weights and the biases, and lets plain gradient descent move weights in single precision, of which the products see a bf16
copy.  Serving quantizes the trained weights once, a scale for each output channel, and every batch of activations as it comes, a scale for each
token; a single token needs no offsets and goes through its expert's weights alone.

    python examples/expert_layers.py [--steps 200]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2210_12415_amd as alt  # noqa: E402


def buffer(size):
    """A workspace as the calls take it; the operators do without one where they ask for none."""
    return dict(workspace=torch.empty(size, dtype=torch.uint8, device="cuda") if size else None, ws_bytes=size)


class Layer:
    """One layer of every expert: y = x w[e]^T + bias[e], with or without ReLU, and its gradients."""

    def __init__(self, handle, rows, experts, inputs, outputs, relu, after_relu, generator):
        self.h, self.after_relu = handle, after_relu
        self.master = torch.randn(experts, outputs, inputs, generator=generator, device="cuda") * inputs ** -0.5
        self.w, self.bias = self.master.bfloat16(), torch.zeros(experts, outputs, device="cuda")
        desc = lambda **kw: alt.grouped_desc(rows, experts, outputs, inputs, **kw)
        self.forward_desc = desc(epilogue=alt.EPI_BIAS | (alt.EPI_RELU if relu else 0))
        self.dx_desc = desc(epilogue=alt.EPI_RELU if after_relu else 0)
        self.dw_desc = desc(out_dtype=alt.F32, epilogue=alt.EPI_BIAS)
        self.y = torch.empty(rows, outputs, dtype=torch.bfloat16, device="cuda")
        self.dx = torch.empty(rows, inputs, dtype=torch.bfloat16, device="cuda")
        self.dw, self.dbias = torch.empty_like(self.master), torch.empty_like(self.bias)
        self.forward_ws = buffer(handle.gemm_grouped_workspace_size(self.forward_desc))
        self.dx_ws = buffer(handle.gemm_grouped_dx_workspace_size(self.dx_desc))
        self.dw_ws = buffer(handle.gemm_grouped_dw_workspace_size(self.dw_desc))

    def forward(self, x, offsets):
        self.x, self.offsets = x, offsets
        self.h.gemm_grouped(self.forward_desc, x, self.w, offsets, self.y, bias=self.bias, **self.forward_ws)
        return self.y

    def by_weights(self, dy):
        self.h.gemm_grouped_dw(self.dw_desc, self.x, dy, self.offsets, self.dw, dbias=self.dbias, **self.dw_ws)

    def by_tokens(self, dy):
        self.h.gemm_grouped_dx(self.dx_desc, dy, self.w, self.offsets, self.dx, relu_of=self.x if self.after_relu else None, **self.dx_ws)
        return self.dx

    def update(self, rate):
        self.master.sub_(self.dw, alpha=rate)
        self.bias.sub_(self.dbias, alpha=rate)
        self.w.copy_(self.master)


class Layer8:
    """A trained layer in 8 bits."""

    def __init__(self, layer, relu):
        self.h, (self.experts, self.outputs, self.inputs) = layer.h, layer.w.shape
        self.w = torch.empty(layer.w.shape, dtype=torch.int8, device="cuda")
        self.scale, self.bias = torch.empty(self.experts, self.outputs, device="cuda"), layer.bias
        self.h.quantize_rows(alt.F32, self.experts * self.outputs, self.inputs, layer.master, self.w, self.scale)
        self.epilogue = alt.EPI_BIAS | (alt.EPI_RELU if relu else 0)

    def quantize(self, x):
        q, scale = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(x.shape[0], device="cuda")
        self.h.quantize_rows(alt.BF16, x.shape[0], x.shape[1], x, q, scale)
        return q, scale

    def batch(self, x, offsets):
        q, scale = self.quantize(x)
        y = torch.empty(x.shape[0], self.outputs, dtype=torch.bfloat16, device="cuda")
        d = alt.grouped_desc(x.shape[0], self.experts, self.outputs, self.inputs, in_dtype=alt.I8, out_dtype=alt.BF16, epilogue=self.epilogue)
        self.h.gemm_grouped(d, q, self.w, offsets, y, a_scale=scale, b_scale=self.scale, bias=self.bias,
                            **buffer(self.h.gemm_grouped_workspace_size(d)))
        return y

    def token(self, x, expert):
        q, scale = self.quantize(x)
        y = torch.empty(1, self.outputs, dtype=torch.bfloat16, device="cuda")
        d = alt.gemm_i8_desc(1, self.outputs, self.inputs, out_dtype=alt.BF16, epilogue=self.epilogue)
        self.h.gemm_i8(d, q, scale, self.w[expert], self.scale[expert], y, bias=self.bias[expert])
        return y


class Block:
    """What the example trains: two layers, and the squared error against another block's answers."""

    def __init__(self, handle, rows, experts, width, hidden, generator):
        self.up = Layer(handle, rows, experts, width, hidden, True, False, generator)
        self.down = Layer(handle, rows, experts, hidden, width, False, True, generator)

    def forward(self, x, offsets):
        return self.down.forward(self.up.forward(x, offsets), offsets)

    def gradients(self, dy):
        self.down.by_weights(dy)
        self.up.by_weights(self.down.by_tokens(dy))

    def step(self, x, offsets, target, rate):
        """One step of gradient descent; returns the loss before it."""
        wrong = self.forward(x, offsets).float() - target
        self.gradients((2 * wrong / wrong.shape[1]).bfloat16())
        for layer in (self.up, self.down):
            layer.update(rate / x.shape[0])
        return float(wrong.square().mean())


class Served:
    def __init__(self, block):
        self.up, self.down = Layer8(block.up, True), Layer8(block.down, False)

    def batch(self, x, offsets):
        return self.down.batch(self.up.batch(x, offsets), offsets)

    def token(self, x, expert):
        return self.down.token(self.up.token(x, expert), expert)


def tokens(counts, width, generator):
    """Tokens sorted by expert, and the first row of each expert."""
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    x = torch.randn(at[-1], width, generator=generator, device="cuda").bfloat16()
    return x, torch.tensor(at, dtype=torch.int32, device="cuda"), at


def main(argv=None):
    p = argparse.ArgumentParser()
    p.add_argument("--steps", type=int, default=200)
    p.add_argument("--width", type=int, default=256)
    p.add_argument("--hidden", type=int, default=1024)
    p.add_argument("--counts", type=int, nargs="+", default=[900, 0, 1500, 333, 1363], help="tokens of each expert")
    p.add_argument("--rate", type=float, default=1.5)
    a = p.parse_args(argv)
    generator, handle = torch.Generator(device="cuda").manual_seed(1), alt.Handle()
    x, offsets, at = tokens(a.counts, a.width, generator)
    teacher, block = (Block(handle, len(x), len(a.counts), a.width, a.hidden, generator) for _ in range(2))
    target = teacher.forward(x, offsets).float()
    losses = [block.step(x, offsets, target, a.rate) for _ in range(a.steps)]
    answer = block.forward(x, offsets).float()
    served = Served(block)
    answer8 = served.batch(x, offsets).float()
    expert = max(range(len(a.counts)), key=lambda e: a.counts[e])
    one = served.token(x[at[expert]:at[expert] + 1], expert).float()
    print("loss %.4f -> %.4f in %d steps; in 8 bits %.4f, answers %.2f %% apart; a single token %s its row of the batch"
          % (losses[0], (answer - target).square().mean(), a.steps, (answer8 - target).square().mean(),
             100 * (answer8 - answer).norm() / answer.norm(), "equals" if torch.equal(one[0], answer8[at[expert]]) else "differs from"))
    return losses


if __name__ == "__main__":
    main()
