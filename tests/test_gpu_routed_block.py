"""The calls around the layers' products in a run together, as a block uses them: forward and every gradient against the same block in 64 bits.

Tolerance, in the 2-norm of each result: every tensor on the way is rounded to bf16, half a step of 2^-8 relative, and passes what it has on; the longest
way from the inputs to a gradient has twelve of them (norm, logits, two layers, the sum; dy times weight, two layers backward, the sum over choices, its
sum with the router's, the norm's gradient, the last sum)."""
import numpy as np
import pytest
import torch

import paper_2210_12415_amd as alt
from examples import routed_block
from rows_util import normal, replayed, ws

pytestmark = pytest.mark.gpu

TOLERANCE = 12 * 2.0 ** -8


def reference(x, block, experts, dy):
    """The block in 64 bits with the experts that it chose: y and the gradients of x, gamma, beta, the router, the experts' layers."""
    t = {"x": x, "gamma": block.norm.gamma, "beta": block.norm.beta, "router": block.router.w[0], "router_bias": block.router.bias[0], "up": block.up.w, "up_bias": block.up.bias,
         "down": block.down.w, "down_bias": block.down.bias}
    t = {k: v.detach().cpu().double().requires_grad_() for k, v in t.items()}
    c = t["x"] - t["x"].mean(1, keepdim=True)
    n = c / torch.sqrt(c.square().mean(1, keepdim=True) + 1e-5) * t["gamma"] + t["beta"]
    logits = n @ t["router"].T + t["router_bias"]
    at = experts.cpu().long()
    weights = torch.softmax(logits.gather(1, at), 1)
    hidden = torch.relu(torch.einsum("tc,tkhc->tkh", n, t["up"][at]) + t["up_bias"][at])
    answers = torch.einsum("tkh,tkch->tkc", hidden, t["down"][at]) + t["down_bias"][at]
    y = t["x"] + (weights[..., None] * answers).sum(1)
    y.backward(dy.cpu().double())
    return y.detach(), {k: v.grad for k, v in t.items()}


def near(got, want, what):
    got, want = got.detach().cpu().double(), want.reshape(got.shape)
    off = float((got - want).norm() / want.norm())
    assert off <= TOLERANCE, (what, off)


@pytest.mark.parametrize("tokens,width,hidden,experts,top", [(300, 128, 192, 8, 2), (77, 72, 40, 5, 3), (1, 64, 64, 4, 1)])
def test_block_and_its_gradients(tokens, width, hidden, experts, top):
    h, g = alt.Handle(), torch.Generator(device="cuda").manual_seed(tokens)
    block = routed_block.RoutedBlock(h, tokens, width, hidden, experts, top, g)
    for v, std, mean in ((block.norm.gamma, 0.2, 1.0), (block.norm.beta, 0.1, 0.0), (block.router.bias, 0.1, 0.0), (block.up.bias, 0.1, 0.0), (block.down.bias, 0.1, 0.0)):
        v.copy_(torch.randn(v.shape, generator=g, device="cuda") * std + mean)
    x, dy = torch.randn(tokens, width, generator=g, device="cuda").bfloat16(), torch.randn(tokens, width, generator=g, device="cuda").bfloat16()
    y = block.forward(x).clone()
    dx = block.gradients(dy)
    torch.cuda.synchronize()
    want, grads = reference(x, block, block.experts, dy)
    near(y, want, "y")
    got = {"x": dx, "gamma": block.norm.dgamma, "beta": block.norm.dbeta, "router": block.router.dw[0], "router_bias": block.router.dbias[0], "up": block.up.dw,
           "up_bias": block.up.dbias, "down": block.down.dw, "down_bias": block.down.dbias}
    for k, v in got.items():
        if tokens > 1 or k not in ("router", "router_bias"):       # (one choice of one: its weight is 1 whatever the logits are)
            near(v, grads[k], k)
    assert int(block.offsets[-1]) == tokens * top


def test_padded_tokens_pass_through_unchanged():
    """Rows of logits that are all -inf: no expert, nothing but the residual, and no part in any gradient but their own."""
    h, g = alt.Handle(), torch.Generator(device="cuda").manual_seed(1)
    tokens, width, experts, top = 40, 64, 6, 2
    d, e = alt.route_desc(tokens, experts, top, dtype=alt.BF16, renormalize=True), alt.exchange_desc(tokens, top, tokens * top, width)
    logits = torch.randn(tokens, experts, generator=g, device="cuda").bfloat16()
    logits[30:] = -float("inf")
    ids, rows = (torch.empty(tokens, top, dtype=torch.int32, device="cuda") for _ in range(2))
    weights, offsets = torch.empty(tokens, top, device="cuda"), torch.empty(experts + 1, dtype=torch.int32, device="cuda")
    h.route(d, logits, ids, weights, rows, offsets, **ws(h.route_workspace_size(d)))
    x, w = torch.randn(tokens, width, generator=g, device="cuda").bfloat16(), torch.randn(experts, width, width, generator=g, device="cuda").bfloat16()
    xe, ye = (torch.full((tokens * top, width), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    h.dispatch_rows(e, x, rows, xe)
    layer = alt.grouped_desc(tokens * top, experts, width, width)
    h.gemm_grouped(layer, xe, w, offsets, ye, **ws(h.gemm_grouped_workspace_size(layer)))
    out = torch.empty_like(x)
    h.combine_rows(e, ye, rows, out, weights=weights)
    assert int(offsets[-1]) == 30 * top and torch.isfinite(out).all() and not out[30:].any() and out[:30].any(1).all()
    dxe, dweights = torch.full_like(xe, float("nan")), torch.empty(tokens, top, device="cuda")
    h.combine_rows_grad(e, x, ye, rows, weights, dxe, dweights)
    dw = torch.empty(experts, width, width, device="cuda")
    d_layer = alt.grouped_desc(tokens * top, experts, width, width, out_dtype=alt.F32)
    h.gemm_grouped_dw(d_layer, xe, dxe, offsets, dw, **ws(h.gemm_grouped_dw_workspace_size(d_layer)))
    dlogits = torch.empty_like(logits)
    h.route_grad(d, logits, ids, dweights, dlogits)
    assert torch.isfinite(dw).all() and torch.isfinite(dlogits).all() and not dlogits[30:].any() and not dweights[30:].any()


def test_block_captured_and_replayed():
    h, g = alt.Handle(), torch.Generator(device="cuda").manual_seed(5)
    block = routed_block.RoutedBlock(h, 500, 128, 192, 8, 2, g)
    x, dy = torch.randn(500, 128, generator=g, device="cuda").bfloat16(), torch.randn(500, 128, generator=g, device="cuda").bfloat16()
    outs = [block.y, block.dx, block.norm.dgamma, block.norm.dbeta, block.router.dw, block.up.dw, block.down.dw, block.dweights, block.offsets]

    def once():
        block.forward(x)
        block.gradients(dy)
    replayed(once, outs, lambda: [o.fill_(2) for o in outs])


def test_two_graphs_share_workspaces():
    """Two captured calls with one workspace, replayed in turn on one stream."""
    h = alt.Handle()
    xs = [normal(i, 900, 512).bfloat16().cuda() for i in (1, 2)]
    d = alt.norm_desc(900, 512)
    space = ws(h.layer_norm_grad_workspace_size(d))
    mean, rstd = torch.empty(900, device="cuda"), torch.empty(900, device="cuda")
    want, graphs, outs = [], [], []
    for x in xs:
        dx, dg, db = torch.empty_like(x), torch.empty(512, device="cuda"), torch.empty(512, device="cuda")

        def once(x=x, dx=dx, dg=dg, db=db):
            h.layer_norm(d, x, dx, mean=mean, rstd=rstd)
            h.layer_norm_grad(d, x, x, mean, rstd, dx, dgamma=dg, dbeta=db, **space)
        once()
        torch.cuda.synchronize()
        want.append([t.clone() for t in (dx, dg, db)])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            once()
        graphs.append(graph)
        outs.append((dx, dg, db))
    for _ in range(3):
        for graph, out, expected in zip(graphs, outs, want):
            for o in out:
                o.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(o, w) for o, w in zip(out, expected))


def test_example_runs_and_serves():
    losses = routed_block.main(["--steps", "3", "--tokens", "200", "--width", "64", "--hidden", "96", "--experts", "5"])
    assert len(losses) == 3 and np.isfinite(losses).all()
