"""What surrounds the products of expert layers in a language model, as cases that can be timed, with their plain forms.

Four kinds of work:

norm       layer norm of rows of `cols` channels:
             mean[m] = sum_c x[m,c] / cols,  rstd[m] = 1 / sqrt(sum_c (x[m,c] - mean[m])^2 / cols + eps),
             y[m,c] = (x[m,c] - mean[m]) * rstd[m] * gamma[c] + beta[c];
           with `train` also mean, rstd and the gradients, from that of y, with u = (x - mean) * rstd and g = dy * gamma:
             dx[m,c] = rstd[m] * (g[m,c] - mean_c(g[m]) - u[m,c] * mean_c(g[m] * u[m])),
             dgamma[c] = sum_m dy[m,c] u[m,c],  dbeta[c] = sum_m dy[m,c].
route      `top` experts for each token, of its logits: score = softmax over the experts, or sigmoid; choice = score + bias where there is a bias, the
           logit itself where there is none.  With groups of experts, a group is worth the sum of the two largest choices in it (scores, without a
           bias), and only the experts of the `top_groups` worthiest groups are chosen from.  The chosen ones come in the order of their choice, ties
           by the lower index; weight = score * scale, divided before by the sum of the chosen scores with `renorm`.  A logit of -inf takes an
           expert out; what a token lacks of `top` experts is expert -1 with weight 0.  rows: the place of each (token, choice) when they are
           ordered by expert, then token, -1 without an expert; offsets: the first place of each expert.  With `train` also the gradient by the logits.
exchange   tokens into the order of their experts and back, n = (token, choice), r = rows[n]:
             xe[r] = x[token],  out[token] = sum_choice weight[n] * ye[r];
           with `train` also the gradients:
             dx[token] = sum_choice dxe[r],  dye[r] = weight[n] * dout[token],  dweight[n] = sum_c dout[token,c] * ye[r,c].
adapters   a projection that all rows share, and beside it the low-rank one of each row's request, g = adapter[m], none where that is -1:
             y[m,n] = sum_k x[m,k] w[n,k] + scale[g] * sum_r (sum_k x[m,k] a[g,r,k]) b[g,n,r] + bias[n].

`own` chooses between the plain forms (elementary torch operations in 32 bits, choices in 64) and the library's operators."""
import math
import random

import torch

own = False

_TYPES = {"bf16": (torch.bfloat16, 2), "f32": (torch.float32, 4)}
_EPS = 1e-5


def listed():
    return [
        # One token each of sixteen sequences in a BERT-shaped layer: latency.
        dict(name="norm_16x768", kind="norm", rows=16, cols=768, dtype="bf16", train=False),
        # A training step of a wide model: what memory gives, and the sums over all rows.
        dict(name="norm_train_16384x4096", kind="norm", rows=16384, cols=4096, dtype="bf16", train=True),
        # Single precision, rows that start at any element.
        dict(name="norm_train_odd_f32", kind="norm", rows=2051, cols=1001, dtype="f32", train=True),
        # Sixteen sequences decoding together, two of 64 experts each.
        dict(name="route_decode", kind="route", tokens=16, experts=64, top=2, dtype="bf16", score="softmax", bias=False, groups=1, top_groups=1, renorm=True,
             padded=0.0, masked=0.0, train=False),
        # A training step: 256 experts in eight groups, a bias that balances them, sigmoid scores.
        dict(name="route_train_256", kind="route", tokens=16384, experts=256, top=8, dtype="f32", score="sigmoid", bias=True, groups=8, top_groups=4,
             renorm=True, padded=0.0, masked=0.0, train=True),
        # A padded batch, a number of experts that fills no wave, some of them barred for some tokens.
        dict(name="route_train_odd", kind="route", tokens=5003, experts=61, top=3, dtype="bf16", score="softmax", bias=False, groups=1, top_groups=1,
             renorm=False, padded=0.2, masked=0.1, train=True),
        # Sixteen sequences decoding together, there and back.
        dict(name="exchange_decode", kind="exchange", tokens=16, experts=64, top=2, cols=2048, dtype="bf16", padded=0.0, train=False),
        # A training step's exchange around a layer of experts.
        dict(name="exchange_train", kind="exchange", tokens=8192, experts=8, top=2, cols=4096, dtype="bf16", padded=0.0, train=True),
        # Single precision, rows that start at any element, tokens without an expert.
        dict(name="exchange_train_odd_f32", kind="exchange", tokens=1501, experts=13, top=3, cols=515, dtype="f32", padded=0.1, train=True),
        # 32 sequences decoding together, each of its own request, through a wide projection: the weights are read once, and little else.
        dict(name="adapters_decode", kind="adapters", M=32, N=4096, K=4096, rank=16, adapters=24, requests=32, bare=4, dtype="bf16", bias=False),
        # Prompts of a dozen requests, a few hundred tokens each.
        dict(name="adapters_prompt", kind="adapters", M=8192, N=4096, K=4096, rank=32, adapters=8, requests=24, bare=2, dtype="bf16", bias=True),
        # Single precision, odd extents.
        dict(name="adapters_odd_f32", kind="adapters", M=333, N=515, K=1030, rank=7, adapters=5, requests=9, bare=1, dtype="f32", bias=True),
    ]


# No drawn case has more work than the largest listed ones.
_MOST_FLOPS, _MOST_BYTES = 2.9e11, 7e8


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _extent(rng, lo, hi):
    """Half of all extents are multiples of 64, as layers have them, the others any number."""
    return max(64, _log(rng, lo, hi) // 64 * 64) if rng.random() < 0.5 else _log(rng, lo, hi)


def draw(rng):
    while True:
        kind = rng.choice(["norm", "route", "exchange", "adapters"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        train = rng.random() < 0.6
        if kind == "norm":
            c = dict(kind=kind, rows=_log(rng, 1, 16384), cols=_extent(rng, 64, 8192), dtype=dtype, train=train)
        elif kind == "route":
            groups = rng.choice([1, 1, 2, 4, 8])
            experts = groups * _log(rng, max(2, 8 // groups), 256 // groups)
            top_groups = rng.randint(1, groups)
            c = dict(kind=kind, tokens=_log(rng, 1, 16384), experts=experts, top=rng.randint(1, min(8, top_groups * experts // groups)), dtype=dtype,
                     score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5, groups=groups, top_groups=top_groups, renorm=rng.random() < 0.5,
                     padded=rng.choice([0.0, 0.2]), masked=rng.choice([0.0, 0.1]), train=train)
        elif kind == "exchange":
            c = dict(kind=kind, tokens=_log(rng, 1, 16384), experts=_log(rng, 8, 256), top=rng.randint(1, 8), cols=_extent(rng, 64, 8192), dtype=dtype,
                     padded=rng.choice([0.0, 0.2]), train=train)
        else:
            m, adapters = _log(rng, 1, 8192), _log(rng, 1, 64)
            requests = min(m, _log(rng, 1, 256))
            c = dict(kind=kind, M=m, N=_extent(rng, 64, 8192), K=_extent(rng, 64, 8192), rank=rng.choice([4, 8, 16, 16, 32, 64, rng.randint(1, 64)]),
                     adapters=adapters, requests=requests, bare=rng.randint(0, requests // 4), dtype=dtype, bias=rng.random() < 0.5)
        w = work(c)
        if w["flops"] <= (_MOST_FLOPS / 8 if dtype == "f32" else _MOST_FLOPS) and w["bytes"] <= _MOST_BYTES:
            return c


def work(case):
    kind, es = case["kind"], _TYPES[case["dtype"]][1]
    if kind == "norm":
        m, c = case["rows"], case["cols"]
        forward = 2 * m * c * es + 8 * c
        if not case["train"]:
            return {"bytes": forward, "flops": 8 * m * c}
        return {"bytes": forward + 8 * m + 3 * m * c * es + 8 * m + 4 * c + 8 * c, "flops": 24 * m * c}
    if kind == "route":
        t, e, k = case["tokens"], case["experts"], case["top"]
        forward = t * e * es + 4 * e * case["bias"] + 12 * t * k + 4 * (e + 1)
        if not case["train"]:
            return {"bytes": forward, "flops": 10 * t * e}
        return {"bytes": forward + 2 * t * e * es + 8 * t * k, "flops": 20 * t * e}
    if kind == "exchange":
        t, k, c = case["tokens"], case["top"], case["cols"]
        n = (t - int(case["padded"] * t)) * k
        forward = (2 * t + 2 * n) * c * es + 12 * t * k
        if not case["train"]:
            return {"bytes": forward, "flops": 2 * n * c}
        return {"bytes": forward + (2 * t + 3 * n) * c * es + 16 * t * k, "flops": 6 * n * c}
    m, n, k, r = case["M"], case["N"], case["K"], case["rank"]
    used = min(case["adapters"], case["requests"] - case["bare"])
    return {"bytes": (m * k + n * k + m * n + used * r * (k + n)) * es + 4 * (m + used + n * case["bias"]), "flops": 2 * m * n * k + 2 * m * r * (n + k)}


# ---- what a program has in hand before the call --------------------------------------------------------------------------

_handle = None


def _library():
    """The package and this program's handle."""
    global _handle
    import paper_2210_12415_amd as alt
    if _handle is None:
        _handle = alt.Handle()
    return alt, _handle


class _Maker:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(int(seed))

    def normal(self, *shape, std=1.0, mean=0.0, dtype=torch.float32):
        """Random normal values; large tensors are drawn in pieces, so that the 32-bit values fit beside them."""
        out = torch.empty(shape, dtype=dtype, device="cuda")
        flat = out.view(-1)
        for at in range(0, flat.numel(), 1 << 26):
            piece = flat[at:at + (1 << 26)]
            piece.copy_(torch.randn(piece.numel(), generator=self.gen, device="cuda").mul_(std).add_(mean))
        return out

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.gen, device="cuda")

    def hidden(self, rows, cols, dtype):
        """A residual stream: channels of different size, some of them far from zero on average."""
        x = torch.randn(rows, cols, generator=self.gen, device="cuda")
        x *= torch.exp(0.5 * torch.randn(cols, generator=self.gen, device="cuda"))
        return x.add_(torch.randn(cols, generator=self.gen, device="cuda")).to(dtype)


def _padding(case, make, tokens):
    """Truth values: tokens that only fill up a batch, a fixed number of them."""
    pad = torch.zeros(tokens, dtype=torch.bool, device="cuda")
    pad[torch.argsort(make.uniform(tokens))[:int(case["padded"] * tokens)]] = True
    return pad


def _adapter_rows(case, seed):
    """The adapter of each row: requests of uneven lengths one after another, each with an adapter of its own choice."""
    rng, m, requests = random.Random(int(seed)), case["M"], case["requests"]
    ids = [i % case["adapters"] for i in range(requests - case["bare"])] + [-1] * case["bare"]
    rng.shuffle(ids)
    share = [rng.uniform(0.3, 1.7) for _ in range(requests)]
    spare, total, rows = m - requests, sum(share), []
    upto = [int(round(spare * sum(share[:i]) / total)) for i in range(requests)] + [spare]
    for i, g in enumerate(ids):
        rows += [g] * (1 + upto[i + 1] - upto[i])
    return rows


def _inputs(case, seed):
    make, kind, dtype = _Maker(seed), case["kind"], _TYPES[case["dtype"]][0]
    s = {}
    if kind == "norm":
        m, c = case["rows"], case["cols"]
        s["x"] = make.hidden(m, c, dtype)
        s["gamma"], s["beta"] = make.normal(c, std=0.2, mean=1.0), make.normal(c, std=0.1)
        if case["train"]:
            s["dy"] = make.normal(m, c, dtype=dtype)
    elif kind == "route":
        t, e = case["tokens"], case["experts"]
        logits = make.normal(t, e) + make.normal(e, std=0.5)
        if case["masked"]:
            logits[make.uniform(t, e) < case["masked"]] = -math.inf
        logits[_padding(case, make, t)] = -math.inf
        s["logits"] = logits.to(dtype)
        s["bias"] = make.normal(e, std=0.02) if case["bias"] else None
        if case["train"]:
            s["dweights"] = make.normal(t, case["top"])
    elif kind == "exchange":
        t, e, k, c = case["tokens"], case["experts"], case["top"], case["cols"]
        popular = make.normal(t, e) + make.normal(e, std=0.5)
        chosen = popular.argsort(1, descending=True)[:, :k]
        pad = _padding(case, make, t)
        chosen = torch.where(pad[:, None], e, chosen).reshape(-1)
        rows = torch.empty(t * k, dtype=torch.int32, device="cuda")
        rows[torch.sort(chosen, stable=True)[1]] = torch.arange(t * k, dtype=torch.int32, device="cuda")
        s["rows"] = torch.where(chosen == e, -1, rows).to(torch.int32).view(t, k)
        s["weights"] = torch.where(pad[:, None], 0.0, make.uniform(t, k) + 0.1)
        s["x"], s["ye"] = make.hidden(t, c, dtype), make.normal(t * k, c, dtype=dtype)
        if case["train"]:
            s["dout"], s["dxe"] = make.normal(t, c, dtype=dtype), make.normal(t * k, c, dtype=dtype)
    else:
        m, n, k, r, g = case["M"], case["N"], case["K"], case["rank"], case["adapters"]
        s["of"] = _adapter_rows(case, seed)
        s["adapter"] = torch.tensor(s["of"], dtype=torch.int32, device="cuda")
        s["x"] = make.normal(m, k, dtype=dtype)
        s["w"] = make.normal(n, k, std=k ** -0.5, dtype=dtype)
        s["a"], s["b"] = make.normal(g, r, k, std=k ** -0.5, dtype=dtype), make.normal(g, n, r, std=0.3 * r ** -0.5, dtype=dtype)
        s["scale"] = make.uniform(g) + 0.5
        s["bias"] = make.normal(n, std=0.1) if case["bias"] else None
    return s


def prepare(case, seed):
    state = {"case": case, "inputs": _inputs(case, seed)}
    if own:
        state["plan"] = _plan(case)
    return state


def _plan(case):
    """Descriptors, output buffers and workspaces, which a program makes once."""
    alt, h = _library()
    kind, dtype = case["kind"], _TYPES[case["dtype"]][0]
    code = {"bf16": alt.BF16, "f32": alt.F32}[case["dtype"]]

    def buffer(*shape, dtype=torch.float32):
        return torch.zeros(shape, dtype=dtype, device="cuda")

    def workspace(need):
        return dict(workspace=torch.empty(need, dtype=torch.uint8, device="cuda") if need else None, ws_bytes=need)

    p = {"alt": alt, "h": h}
    if kind == "norm":
        m, c = case["rows"], case["cols"]
        p["d"] = alt.norm_desc(m, c, in_dtype=code, out_dtype=code, eps=_EPS)
        p["y"] = buffer(m, c, dtype=dtype)
        if case["train"]:
            p["mean"], p["rstd"], p["dx"], p["dgamma"], p["dbeta"] = buffer(m), buffer(m), buffer(m, c, dtype=dtype), buffer(c), buffer(c)
            p["ws"] = workspace(h.layer_norm_grad_workspace_size(p["d"]))
    elif kind == "route":
        t, e, k = case["tokens"], case["experts"], case["top"]
        p["d"] = alt.route_desc(t, e, k, dtype=code, score=alt.SCORE_SOFTMAX if case["score"] == "softmax" else alt.SCORE_SIGMOID, groups=case["groups"],
                                top_groups=case["top_groups"], group_best=2, renormalize=case["renorm"], scale=_SCALE)
        p["experts"], p["rows"], p["offsets"] = (buffer(*n, dtype=torch.int32) for n in ((t, k), (t, k), (e + 1,)))
        p["weights"] = buffer(t, k)
        p["ws"] = workspace(h.route_workspace_size(p["d"]))
        if case["train"]:
            p["dlogits"] = buffer(t, e, dtype=dtype)
    elif kind == "exchange":
        t, k, c = case["tokens"], case["top"], case["cols"]
        p["d"] = alt.exchange_desc(t, k, t * k, c, dtype=code)
        p["xe"], p["out"] = buffer(t * k, c, dtype=dtype), buffer(t, c, dtype=dtype)
        if case["train"]:
            p["dx"], p["dye"], p["dweights"] = buffer(t, c, dtype=dtype), buffer(t * k, c, dtype=dtype), buffer(t, k)
    else:
        p["d"] = alt.adapters_desc(case["M"], case["N"], case["K"], case["adapters"], case["rank"], in_dtype=code, out_dtype=code,
                                   epilogue=alt.EPI_BIAS if case["bias"] else 0)
        p["y"] = buffer(case["M"], case["N"], dtype=dtype)
        p["ws"] = workspace(h.gemm_adapters_workspace_size(p["d"]))
    return p


# ---- one pass ------------------------------------------------------------------------------------------------------------

# What the routed weights are multiplied by.
_SCALE = 1.5


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    case, s, p = state["case"], state["inputs"], state["plan"]
    h, kind = p["h"], case["kind"]
    if kind == "norm":
        if not case["train"]:
            h.layer_norm(p["d"], s["x"], p["y"], gamma=s["gamma"], beta=s["beta"])
            return p["y"]
        h.layer_norm(p["d"], s["x"], p["y"], gamma=s["gamma"], beta=s["beta"], mean=p["mean"], rstd=p["rstd"])
        h.layer_norm_grad(p["d"], s["dy"], s["x"], p["mean"], p["rstd"], p["dx"], gamma=s["gamma"], dgamma=p["dgamma"], dbeta=p["dbeta"], **p["ws"])
        return tuple(p[n] for n in ("y", "mean", "rstd", "dx", "dgamma", "dbeta"))
    if kind == "route":
        h.route(p["d"], s["logits"], p["experts"], p["weights"], p["rows"], p["offsets"], bias=s["bias"], **p["ws"])
        out = tuple(p[n] for n in ("experts", "weights", "rows", "offsets"))
        if not case["train"]:
            return out
        h.route_grad(p["d"], s["logits"], p["experts"], s["dweights"], p["dlogits"])
        return out + (p["dlogits"],)
    if kind == "exchange":
        h.dispatch_rows(p["d"], s["x"], s["rows"], p["xe"])
        h.combine_rows(p["d"], s["ye"], s["rows"], p["out"], weights=s["weights"])
        if not case["train"]:
            return p["xe"], p["out"]
        h.combine_rows_grad(p["d"], s["dout"], s["ye"], s["rows"], s["weights"], p["dye"], p["dweights"])
        h.combine_rows(p["d"], s["dxe"], s["rows"], p["dx"])
        return tuple(p[n] for n in ("xe", "out", "dx", "dye", "dweights"))
    h.gemm_adapters(p["d"], s["x"], s["w"], s["adapter"], s["a"], s["b"], p["y"], scale=s["scale"], bias=s["bias"], **p["ws"])
    return p["y"]


def _run_plain(state):
    return {"norm": _norm_plain, "route": _route_plain, "exchange": _exchange_plain, "adapters": _adapters_plain}[state["case"]["kind"]](
        state["case"], state["inputs"])


def _norm_plain(case, s):
    dtype = _TYPES[case["dtype"]][0]
    x = s["x"].float()
    mean = x.mean(1)
    centred = x - mean[:, None]
    rstd = 1 / ((centred * centred).mean(1) + _EPS).sqrt()
    u = centred * rstd[:, None]
    y = (u * s["gamma"] + s["beta"]).to(dtype)
    if not case["train"]:
        return y
    dy = s["dy"].float()
    g = dy * s["gamma"]
    dx = rstd[:, None] * (g - g.mean(1)[:, None] - u * (g * u).mean(1)[:, None])
    return y, mean, rstd, dx.to(dtype), (dy * u).sum(0), dy.sum(0)


def _best(values):
    """Largest value of each row and the first index that holds it."""
    top = values.amax(-1)
    index = torch.arange(values.shape[-1], device=values.device)
    return top, torch.where(values == top[..., None], index, values.shape[-1]).amin(-1).clamp_(max=values.shape[-1] - 1)


def _route_plain(case, s):
    t, e, k, groups = case["tokens"], case["experts"], case["top"], case["groups"]
    l = s["logits"].double()
    there = l > -math.inf
    if case["score"] == "softmax":
        top = torch.where(there.any(1), l.amax(1), 0.0)
        score = (l - top[:, None]).exp()
        score = score / score.sum(1).clamp_(min=1e-300)[:, None]
    else:
        score = 1 / (1 + (-l).exp())
    worth = score + s["bias"].double() if case["bias"] else score
    worth = torch.where(there, worth, -math.inf)
    choice = worth if case["bias"] else l
    if groups > 1:
        left = worth.view(t, groups, e // groups)
        total = torch.full((t, groups), -math.inf, dtype=torch.float64, device=l.device)
        for i in range(min(2, e // groups)):
            top, at = _best(left)
            total = torch.where(top > -math.inf, top if i == 0 else total + top, total)
            left = left.scatter(2, at[..., None], -math.inf)
        kept = torch.zeros_like(total, dtype=torch.bool)
        for _ in range(case["top_groups"]):
            top, at = _best(total)
            kept = kept.scatter(1, at[:, None], True)
            total = total.scatter(1, at[:, None], -math.inf)
        choice = torch.where(kept[..., None], choice.view(t, groups, e // groups), -math.inf).view(t, e)
    experts, weights = [], []
    for _ in range(k):
        top, at = _best(choice)
        has = top > -math.inf
        experts.append(torch.where(has, at, -1))
        weights.append(torch.where(has, score.gather(1, at[:, None])[:, 0], 0.0))
        choice = choice.scatter(1, at[:, None], -math.inf)
    experts, chosen = torch.stack(experts, 1), torch.stack(weights, 1)
    total = chosen.sum(1, keepdim=True)
    total = torch.where(total > 0, total, 1.0)
    weights = _SCALE * (chosen / total if case["renorm"] else chosen)
    flat = torch.where(experts < 0, e, experts).reshape(-1)
    order = torch.sort(flat, stable=True)[1]
    rows = torch.empty_like(order)
    rows[order] = torch.arange(t * k, device=l.device)
    rows = torch.where(flat == e, -1, rows).view(t, k).to(torch.int32)
    counts = (experts.reshape(-1, 1) == torch.arange(e, device=l.device)).sum(0)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
    out = experts.to(torch.int32), weights.float(), rows, offsets
    if not case["train"]:
        return out
    has = experts >= 0
    dw = torch.where(has, s["dweights"].double(), 0.0) * _SCALE
    ds = (dw - (dw * chosen / total).sum(1, keepdim=True)) / total if case["renorm"] else dw
    ds = torch.zeros_like(score).scatter_add(1, experts.clamp(min=0), torch.where(has, ds, 0.0))
    if case["score"] == "softmax":
        dl = score * (ds - (ds * score).sum(1, keepdim=True))
    else:
        dl = ds * score * (1 - score)
    return out + (dl.to(s["logits"].dtype),)


def _exchange_plain(case, s):
    t, k, c, dtype = case["tokens"], case["top"], case["cols"], _TYPES[case["dtype"]][0]
    rows = s["rows"].long()
    there, at = rows >= 0, rows.clamp(min=0)
    xe = torch.zeros(t * k + 1, c, dtype=dtype, device="cuda")
    out = torch.zeros(t, c, device="cuda")
    if case["train"]:
        dye = torch.zeros(t * k + 1, c, dtype=dtype, device="cuda")
        dx, dweights, dout = torch.zeros(t, c, device="cuda"), [], s["dout"].float()
    for j in range(k):
        to, has = torch.where(there[:, j], rows[:, j], t * k), there[:, j, None]
        w = s["weights"][:, j, None]
        y = torch.where(has, s["ye"][at[:, j]].float(), 0.0)
        xe[to] = s["x"]
        out += w * y
        if case["train"]:
            dye[to] = (w * dout).to(dtype)
            dx += torch.where(has, s["dxe"][at[:, j]].float(), 0.0)
            dweights.append((dout * y).sum(1))
    if not case["train"]:
        return xe[:t * k], out.to(dtype)
    return xe[:t * k], out.to(dtype), dx.to(dtype), dye[:t * k], torch.stack(dweights, 1)


def _runs(of):
    """(first row, end, adapter) of each run of rows with one adapter."""
    first = 0
    for m in range(1, len(of) + 1):
        if m == len(of) or of[m] != of[first]:
            yield first, m, of[first]
            first = m


def _adapters_plain(case, s):
    x = s["x"].float()
    y = torch.matmul(x, s["w"].float().t())
    for lo, hi, g in _runs(s["of"]):
        if g >= 0:
            down = torch.matmul(x[lo:hi], s["a"][g].float().t())
            y[lo:hi] += s["scale"][g] * torch.matmul(down, s["b"][g].float().t())
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(_TYPES[case["dtype"]][0])


# ---- the definition, in 64 bits -------------------------------------------------------------------------------------------

def exact(case, seed):
    return {"norm": _norm_exact, "route": _route_exact, "exchange": _exchange_exact, "adapters": _adapters_exact}[case["kind"]](case, _inputs(case, seed))


def _norm_exact(case, s):
    x = s["x"].to(torch.float64)
    n = x.shape[1]
    mean = x.sum(dim=1, keepdim=True) / n
    x -= mean
    rstd = torch.pow(x.square().sum(dim=1, keepdim=True) / n + _EPS, -0.5)
    x *= rstd
    y = torch.addcmul(s["beta"].double(), x, s["gamma"].double())
    if not case["train"]:
        return y
    dy = s["dy"].to(torch.float64)
    dbeta, dgamma = torch.ones(x.shape[0], dtype=torch.float64, device="cuda") @ dy, torch.einsum("mc,mc->c", dy, x)
    g = dy.mul_(s["gamma"].double())
    along = torch.einsum("mc,mc->m", g, x).div_(n).unsqueeze(1)
    return y, mean.squeeze(1), rstd.squeeze(1), rstd * (g - g.sum(dim=1, keepdim=True) / n - x * along), dgamma, dbeta


def _route_exact(case, s):
    """By a full stable sort of the choices."""
    tokens, experts, top, groups = case["tokens"], case["experts"], case["top"], case["groups"]
    logits = s["logits"].double()
    barred = torch.isneginf(logits)
    score = torch.sigmoid(logits) if case["score"] == "sigmoid" else torch.nan_to_num(torch.softmax(logits, dim=1), nan=0.0)
    worth = score if s["bias"] is None else score + s["bias"].double().unsqueeze(0)
    key = (logits if s["bias"] is None else worth).masked_fill(barred, -math.inf)
    if groups > 1:
        inside = worth.masked_fill(barred, -math.inf).unflatten(1, (groups, -1)).sort(dim=2, descending=True)[0][:, :, :2]
        value = torch.nan_to_num(inside, neginf=0.0).sum(dim=2).masked_fill(torch.isneginf(inside[:, :, 0]), -math.inf)
        place = value.sort(dim=1, descending=True, stable=True)[1].argsort(dim=1)
        key = key.masked_fill((place >= case["top_groups"]).repeat_interleave(experts // groups, dim=1), -math.inf)
    ordered, index = key.sort(dim=1, descending=True, stable=True)
    none = torch.isneginf(ordered[:, :top])
    pick = index[:, :top]
    raw = score.gather(1, pick).masked_fill(none, 0.0)
    weights = raw * _SCALE
    if case["renorm"]:
        weights = weights / raw.sum(dim=1, keepdim=True).masked_fill(none[:, :1], 1.0)
    pick = pick.masked_fill(none, -1)
    flat = pick.flatten()
    taken = flat >= 0
    counts = torch.bincount(flat[taken], minlength=experts)
    offsets = torch.zeros(experts + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = counts.cumsum(dim=0)
    rows = torch.full_like(flat, -1)
    where = taken.nonzero().squeeze(1)
    rows[where[flat[where].argsort(stable=True)]] = torch.arange(where.numel(), device="cuda")
    out = (pick.int(), weights, rows.view(tokens, top).int(), offsets.int())
    if not case["train"]:
        return out
    # the gradient, through the derivatives of each chosen weight by each chosen score and of each score by the logits
    up = s["dweights"].double().masked_fill(none, 0.0)
    if case["renorm"]:
        share = weights / _SCALE
        up = (up - (up * share).sum(dim=1, keepdim=True)) / raw.sum(dim=1, keepdim=True).masked_fill(none[:, :1], 1.0)
    up = (up * _SCALE).masked_fill(none, 0.0)
    dlogits = torch.zeros_like(score)
    slot = pick.clamp(min=0)
    if case["score"] == "sigmoid":
        dlogits.scatter_add_(1, slot, up * raw * (1.0 - raw))
    else:
        dlogits -= score * (up * raw).sum(dim=1, keepdim=True)
        dlogits.scatter_add_(1, slot, up * raw)
    return out + (dlogits,)


def _exchange_exact(case, s):
    tokens, top, cols = case["tokens"], case["top"], case["cols"]
    flat = s["rows"].flatten().long()
    slots = (flat >= 0).nonzero().squeeze(1)
    token, row = slots // top, flat[slots]
    w = s["weights"].flatten().double()[slots].unsqueeze(1)
    xe = torch.zeros(tokens * top, cols, dtype=torch.float64, device="cuda")
    xe[row] = s["x"].double()[token]
    out = torch.zeros(tokens, cols, dtype=torch.float64, device="cuda")
    picked = s["ye"].double()[row]
    out.index_add_(0, token, w * picked)
    if not case["train"]:
        return xe, out
    dx = torch.zeros_like(out).index_add_(0, token, s["dxe"].double()[row])
    up = s["dout"].double()[token]
    dweights = torch.zeros(tokens * top, dtype=torch.float64, device="cuda")
    dweights[slots] = (up * picked).sum(dim=1)
    dye = torch.zeros_like(xe)
    dye[row] = w * up
    return xe, out, dx, dye, dweights.view(tokens, top)


def _adapters_exact(case, s):
    x = s["x"].double()
    y = x @ s["w"].double().T
    for g in sorted(set(s["of"]) - {-1}):
        mine = (s["adapter"] == g).nonzero().squeeze(1)
        y[mine] += s["scale"][g].double() * ((x[mine] @ s["a"][g].double().T) @ s["b"][g].double().T)
    return y if s["bias"] is None else y + s["bias"].double()
