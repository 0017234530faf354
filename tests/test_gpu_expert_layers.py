"""The example that trains a block of experts and serves it in 8 bits, against the same block in 64 bits."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))
import paper_2210_12415_amd as alt  # noqa: E402
import expert_layers as ex  # noqa: E402

pytestmark = pytest.mark.gpu

COUNTS, WIDTH, HIDDEN = [70, 0, 1, 129, 40], 96, 200
BF16, EPS = 2.0 ** -8, 2.0 ** -24


def block():
    g = torch.Generator(device="cuda").manual_seed(3)
    x, offsets, at = ex.tokens(COUNTS, WIDTH, g)
    b = ex.Block(alt.Handle(), len(x), len(COUNTS), WIDTH, HIDDEN, g)
    for layer in (b.up, b.down):
        layer.bias.normal_(generator=g)
    return b, x, offsets, at, g


def test_gradients_of_a_block():
    """Against autograd in 64 bits.  Every tensor between the products is rounded to bf16 once (2^-8 of the value, the sums' own error included);
    what an error does downstream is bounded by the magnitudes that it meets there: |A|, |dy| and |w| in place of A, dy and w."""
    b, x, offsets, at, g = block()
    y = b.forward(x, offsets)
    dy = torch.randn(y.shape, generator=g, device="cuda").bfloat16()
    b.gradients(dy)
    torch.cuda.synchronize()
    for e in range(len(COUNTS)):
        lo, hi = at[e], at[e + 1]
        w1, w2, b1, b2 = (t[e].double().cpu().requires_grad_() for t in (b.up.w, b.down.w, b.up.bias, b.down.bias))
        xe, dye = x[lo:hi].double().cpu(), dy[lo:hi].double().cpu()
        # (the ReLU's own gradient is taken where the kernels' rounded values have it: the test's inputs leave none within a rounding of zero)
        hid = torch.relu(xe @ w1.T + b1)
        out = hid @ w2.T + b2
        out.backward(dye)
        h_err = BF16 * hid.detach()
        y_err = h_err @ w2.detach().abs().T + BF16 * out.detach().abs() + HIDDEN * EPS * (hid.detach() @ w2.detach().abs().T + b2.detach().abs())
        assert bool(((y[lo:hi].double().cpu() - out.detach()).abs() <= y_err + 1e-6).all())
        got = hid.detach() > 0
        assert torch.equal(got, b.up.y[lo:hi].cpu() > 0)
        dh_abs = (dye.abs() @ w2.detach().abs()) * got
        dh_err = BF16 * ((dye @ w2.detach()).abs() * got) + WIDTH * EPS * dh_abs
        rows = (hi - lo) * EPS
        bounds = ((b.down.dw, w2.grad, dye.abs().T @ h_err + rows * (dye.abs().T @ hid.detach())),
                  (b.down.dbias, b2.grad, rows * dye.abs().sum(0)),
                  (b.up.dw, w1.grad, dh_err.T @ xe.abs() + rows * (dh_abs.T @ xe.abs())),
                  (b.up.dbias, b1.grad, dh_err.sum(0) + rows * dh_abs.sum(0)))
        for own, want, bound in bounds:
            assert bool(((own[e].double().cpu() - want).abs() <= 1.01 * bound + 1e-9).all())


def test_training_lowers_the_loss():
    losses = ex.main(["--steps", "12", "--width", "64", "--hidden", "128", "--counts", "100", "0", "57", "43", "--rate", "1"])
    assert all(later < before for before, later in zip(losses, losses[1:]))


def test_served_in_8_bits():
    """Against the float block: each operand is off by half its scale at most, each layer's output by a bf16 rounding."""
    b, x, offsets, at, g = block()
    served = ex.Served(b)
    y = served.batch(x, offsets)
    torch.cuda.synchronize()

    def layer(v, v_err, l, l8, e, relu):
        """Value and bound of the error of a layer, in 64 bits, of inputs v that are off by v_err."""
        w, bias, t = l.master[e].double().cpu(), l.bias[e].double().cpu(), l8.scale[e].double().cpu()
        most = v.abs() + v_err
        s = most.amax(1, keepdim=True) / 127 * (1 + 2.0 ** -15)
        off = (v_err + s / 2) @ w.abs().T + (most + s / 2).sum(1, keepdim=True) * t / 2
        out = v @ w.T + bias
        return (torch.relu(out) if relu else out), off + (out.abs() + off) * (BF16 + 8 * EPS)

    for e in range(len(COUNTS)):
        lo, hi = at[e], at[e + 1]
        if hi == lo:
            continue
        v = x[lo:hi].double().cpu()
        hid, h_err = layer(v, torch.zeros_like(v), b.up, served.up, e, True)
        want, err = layer(hid, h_err, b.down, served.down, e, False)
        got = y[lo:hi].double().cpu()
        assert bool(((got - want).abs() <= err).all())
        # sums of 8-bit products are exact: a token alone gives the bits that it gives in the batch
        assert torch.equal(served.token(x[lo:lo + 1], e)[0], y[lo])
