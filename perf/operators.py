"""Products of expert layers and of 8-bit layers, as cases that can be timed, with their plain forms.

Three kinds of work:

quantize   rows of activations to 8 bits with a scale for each row (token):
             s[m] = max_k |x[m,k]| / 127, rounded up to 16 significant bits and at least 2^-126,  q[m,k] = round(x[m,k] / s[m]), ties to even.
           (A scale of 16 bits makes q * s exact in 32 bits, so that q has one right value.)  The pass returns q * s and s.
product8   y[m,n] = sum_k q[m,k] w[n,k] * s[m] * t[n] + bias[n], q and w in 8 bits, s for each token, t for each output channel; with
           `quantize` the pass begins at the activations and quantizes them first, as a serving program does.
experts    rows of tokens in the order of their experts, expert e owning rows [offsets[e], offsets[e+1]):
             y[m,n] = sum_k x[m,k] w[e,n,k] + bias[e,n], with or without ReLU;
           in 8 bits as above; with `train` also the gradients of x (through the ReLU that made x), w and bias from that of y:
             dx[m,k] = [x[m,k] > 0] sum_n dy[m,n] w[e,n,k],  dw[e,n,k] = sum_{m of e} dy[m,n] x[m,k],  db[e,n] = sum_{m of e} dy[m,n].

`own` chooses between the plain forms (elementary torch operations in 32 bits) and the library's operators."""
import math
import random

import torch

own = False

_TYPES = {"bf16": (torch.bfloat16, 2), "f32": (torch.float32, 4), "i8": (torch.int8, 1)}


def listed():
    return [
        # One sequence of 128 tokens of a BERT-shaped layer on its way into an 8-bit product: latency.
        dict(name="quantize_128x768", kind="quantize", rows=128, cols=768, dtype="bf16"),
        # A large batch of prompts: what memory gives.
        dict(name="quantize_16384x4096", kind="quantize", rows=16384, cols=4096, dtype="bf16"),
        # One token of the same layer's feed-forward up: both calls are launch latency.
        dict(name="product8_one_token", kind="product8", M=1, N=3072, K=768, out="bf16", bias=True, relu=True, quantize=True),
        # Sixteen sequences decoding together through a wide layer: the weights are read once, and little else.
        dict(name="product8_decode", kind="product8", M=16, N=8192, K=8192, out="bf16", bias=False, relu=False, quantize=False),
        # Odd extents: rows that start at any byte, tiles that end early.
        dict(name="product8_odd", kind="product8", M=333, N=1001, K=2049, out="f32", bias=True, relu=False, quantize=False),
        # Feed-forward down of the BERT-shaped layer over 16 sequences of 128 tokens.
        dict(name="product8_ffn_down", kind="product8", M=2048, N=768, K=3072, out="bf16", bias=True, relu=False, quantize=True),
        # A large prompt batch: the matrix cores.
        dict(name="product8_8192", kind="product8", M=8192, N=8192, K=8192, out="bf16", bias=False, relu=False, quantize=False),
        # Eight tokens with two experts each: most experts have one row or none, and the chosen ones' weights are read once.
        dict(name="experts_decode", kind="experts", rows=16, groups=64, N=2048, K=1024, dtype="bf16", skew=0.0, empty=50, bias=True, relu=True, train=False,
             quantize=False),
        # The same in 8 bits, more tokens and larger experts.
        dict(name="experts_decode_i8", kind="experts", rows=64, groups=32, N=4096, K=2048, dtype="i8", skew=1.0, empty=4, bias=False, relu=False, train=False,
             quantize=True),
        # Prompts through experts in 8 bits, some of them far more popular than others.
        dict(name="experts_prompt_i8", kind="experts", rows=16384, groups=32, N=4096, K=2048, dtype="i8", skew=0.7, empty=1, bias=True, relu=True, train=False,
             quantize=False),
        # A training step's second expert product: forward, and the three gradients.
        dict(name="experts_train", kind="experts", rows=16384, groups=8, N=2048, K=4096, dtype="bf16", skew=0.3, empty=0, bias=True, relu=False, train=True,
             quantize=False),
        # Single precision, odd extents, an expert without a token.
        dict(name="experts_train_odd_f32", kind="experts", rows=1001, groups=13, N=515, K=1030, dtype="f32", skew=1.2, empty=1, bias=True, relu=False, train=True,
             quantize=False),
    ]


# No drawn case has more work than the largest listed ones.
_MOST_FLOPS, _MOST_BYTES = 8e11, 8e8


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _extent(rng, lo, hi):
    """Half of all extents are multiples of 64, as layers have them, the others any number."""
    return max(64, _log(rng, lo, hi) // 64 * 64) if rng.random() < 0.5 else _log(rng, lo, hi)


def draw(rng):
    while True:
        kind = rng.choice(["quantize", "product8", "product8", "experts", "experts", "experts"])
        if kind == "quantize":
            c = dict(kind=kind, rows=_log(rng, 1, 16384), cols=_extent(rng, 64, 8192), dtype=rng.choice(["bf16", "f32"]))
        elif kind == "product8":
            c = dict(kind=kind, M=_log(rng, 1, 8192), N=_extent(rng, 64, 8192), K=_extent(rng, 64, 8192), out=rng.choice(["bf16", "f32"]),
                     bias=rng.random() < 0.5, relu=rng.random() < 0.5, quantize=rng.random() < 0.5)
        else:
            dtype = rng.choice(["bf16", "bf16", "i8", "f32"])
            groups = _log(rng, 1, 64)
            c = dict(kind=kind, rows=_log(rng, 1, 16384), groups=groups, N=_extent(rng, 64, 4096), K=_extent(rng, 64, 4096), dtype=dtype,
                     skew=round(rng.uniform(0.0, 1.5), 2), empty=rng.randrange(0, groups), bias=rng.random() < 0.5, relu=rng.random() < 0.5,
                     train=dtype != "i8" and rng.random() < 0.6, quantize=dtype == "i8" and rng.random() < 0.5)
            if c["train"]:
                c["relu"], c["bias"] = False, True
        w = work(c)
        limit = _MOST_FLOPS / 4 if c.get("dtype") == "f32" else _MOST_FLOPS
        if w["flops"] <= limit and w["bytes"] <= _MOST_BYTES:
            return c


def _counts(case):
    """Rows of each expert, most popular first: shares fall as a power of the rank; the last `empty` experts have none."""
    active = max(1, case["groups"] - case["empty"])
    share = [(i + 1.0) ** -case["skew"] for i in range(active)]
    total, rows = sum(share), case["rows"]
    upto = [int(round(rows * sum(share[:i]) / total)) for i in range(active)] + [rows]
    return [upto[i + 1] - upto[i] for i in range(active)] + [0] * (case["groups"] - active)


def work(case):
    kind = case["kind"]
    if kind == "quantize":
        m, k = case["rows"], case["cols"]
        return {"bytes": m * k * (_TYPES[case["dtype"]][1] + 1) + 4 * m, "flops": 3 * m * k}
    if kind == "product8":
        m, n, k = case["M"], case["N"], case["K"]
        return {"bytes": m * k * (2 if case["quantize"] else 1) + n * k + 4 * (m + n + n * case["bias"]) + m * n * _TYPES[case["out"]][1],
                "flops": 2 * m * n * k}
    counts = _counts(case)
    m, n, k, e = case["rows"], case["N"], case["K"], sum(c > 0 for c in counts)
    es = _TYPES[case["dtype"]][1]
    os = 4 if case["dtype"] == "f32" else 2
    forward = m * k * (2 if case["quantize"] else es) + e * n * k * es + m * n * os + 4 * e * n * case["bias"]
    if case["dtype"] == "i8":
        forward += 4 * (m + e * n)
    if not case["train"]:
        return {"bytes": forward, "flops": 2 * m * n * k}
    # dx reads dy, w and the sign of x and writes dx; dw reads dy and x and writes the whole of dw in 32 bits
    dx = m * n * es + e * n * k * es + 2 * m * k * es
    dw = m * n * es + m * k * es + 4 * case["groups"] * n * k + 4 * case["groups"] * n
    return {"bytes": forward + dx + dw, "flops": 6 * m * n * k}


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

    def normal(self, *shape, std=1.0, dtype=torch.float32):
        """Random normal values; large tensors are drawn in pieces, so that the 32-bit values fit beside them."""
        out = torch.empty(shape, dtype=dtype, device="cuda")
        flat = out.view(-1)
        for at in range(0, flat.numel(), 1 << 26):
            piece = flat[at:at + (1 << 26)]
            piece.copy_(torch.randn(piece.numel(), generator=self.gen, device="cuda").mul_(std))
        return out

    def activations(self, rows, cols, dtype, after_relu=False):
        """Normal values whose channels differ in size, some by a lot, as they do behind a norm's gain."""
        x = torch.randn(rows, cols, generator=self.gen, device="cuda")
        x *= torch.exp(0.5 * torch.randn(cols, generator=self.gen, device="cuda"))
        if after_relu:
            x.clamp_(min=0)
        return x.to(dtype)

    def weights8(self, *shape):
        """Weights in 8 bits with a scale for each output channel."""
        w = torch.empty(shape, dtype=torch.int8, device="cuda")
        t = torch.empty(shape[:-1], dtype=torch.float32, device="cuda")
        for part, scale in zip(w.view(-1, *shape[-2:]), t.view(-1, shape[-2])):
            v = torch.randn(shape[-2:], generator=self.gen, device="cuda").mul_(shape[-1] ** -0.5)
            scale.copy_(v.abs().amax(1).clamp_(min=1e-20) / 127)
            part.copy_((v / scale[:, None]).round_().clamp_(-127, 127))
        return w, t


def _offsets(case, seed):
    """First row of each expert and, last, the number of rows; which expert is popular differs from seed to seed."""
    counts = _counts(case)
    random.Random(int(seed)).shuffle(counts)
    at = [0]
    for c in counts:
        at.append(at[-1] + c)
    return at


def _inputs(case, seed):
    make, kind = _Maker(seed), case["kind"]
    if kind == "quantize":
        return dict(x=make.activations(case["rows"], case["cols"], _TYPES[case["dtype"]][0]))
    s = {}
    if kind == "product8":
        m, n, k, lead = case["M"], case["N"], case["K"], ()
    else:
        m, n, k, lead = case["rows"], case["N"], case["K"], (case["groups"],)
        s["at"] = _offsets(case, seed)
        s["offsets"] = torch.tensor(s["at"], dtype=torch.int32, device="cuda")
    if kind == "product8" or case["dtype"] == "i8":
        s["x"] = make.activations(m, k, torch.bfloat16)
        s["w"], s["t"] = make.weights8(*lead, n, k)
        if not case["quantize"]:
            s["q"], s["s"] = _quantize(s.pop("x"))
    else:
        dtype = _TYPES[case["dtype"]][0]
        s["x"] = make.activations(m, k, dtype, after_relu=case["train"])
        s["w"] = make.normal(*lead, n, k, std=k ** -0.5, dtype=dtype)
        if case["train"]:
            s["dy"] = make.normal(m, n, dtype=dtype)
    s["bias"] = make.normal(*lead, n, std=0.1) if case["bias"] else None
    return s


def prepare(case, seed):
    state = {"case": case, "inputs": _inputs(case, seed)}
    if own:
        state["plan"] = _plan(case)
    return state


def _plan(case):
    """Descriptors, output buffers and workspace, which a program makes once."""
    alt, h = _library()
    kind = case["kind"]

    def empty(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda")

    p = {"alt": alt, "h": h}
    if kind == "quantize":
        p["in"] = alt.BF16 if case["dtype"] == "bf16" else alt.F32
        p["q"], p["s"] = empty(case["rows"], case["cols"], dtype=torch.int8), empty(case["rows"])
        return p
    m, n, k = case["M" if kind == "product8" else "rows"], case["N"], case["K"]
    epilogue = (alt.EPI_BIAS if case["bias"] else 0) | (alt.EPI_RELU if case["relu"] else 0)
    if case["quantize"]:
        p["q"], p["s"] = empty(m, k, dtype=torch.int8), empty(m)
    if kind == "product8":
        out = case["out"]
        p["d"] = alt.gemm_i8_desc(m, n, k, out_dtype=alt.BF16 if out == "bf16" else alt.F32, epilogue=epilogue)
        need = h.gemm_i8_workspace_size(p["d"])
    else:
        out = "f32" if case["dtype"] == "f32" else "bf16"
        code = {"bf16": alt.BF16, "f32": alt.F32, "i8": alt.I8}[case["dtype"]]
        o = alt.BF16 if out == "bf16" else alt.F32
        p["d"] = alt.grouped_desc(m, case["groups"], n, k, in_dtype=code, out_dtype=o, epilogue=epilogue)
        need = h.gemm_grouped_workspace_size(p["d"])
        if case["train"]:
            p["d_dx"] = alt.grouped_desc(m, case["groups"], n, k, in_dtype=code, out_dtype=o, epilogue=alt.EPI_RELU)
            p["d_dw"] = alt.grouped_desc(m, case["groups"], n, k, in_dtype=code, out_dtype=alt.F32, epilogue=alt.EPI_BIAS)
            need = max(need, h.gemm_grouped_dx_workspace_size(p["d_dx"]), h.gemm_grouped_dw_workspace_size(p["d_dw"]))
            p["dx"] = empty(m, k, dtype=_TYPES[out][0])
            p["dw"], p["db"] = empty(case["groups"], n, k), empty(case["groups"], n)
    p["y"] = empty(m, n, dtype=_TYPES[out][0])
    p["ws"] = dict(workspace=empty(need, dtype=torch.uint8) if need else None, ws_bytes=need)
    return p


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    case, s, p = state["case"], state["inputs"], state["plan"]
    alt, h = p["alt"], p["h"]
    if case["kind"] == "quantize":
        h.quantize_rows(p["in"], case["rows"], case["cols"], s["x"], p["q"], p["s"])
        return p["q"] * p["s"][:, None], p["s"]
    q, scale = s.get("q"), s.get("s")
    if case["quantize"]:
        q, scale = p["q"], p["s"]
        h.quantize_rows(alt.BF16, s["x"].shape[0], s["x"].shape[1], s["x"], q, scale)
    if case["kind"] == "product8":
        h.gemm_i8(p["d"], q, scale, s["w"], s["t"], p["y"], bias=s["bias"], **p["ws"])
        return p["y"]
    if case["dtype"] == "i8":
        h.gemm_grouped(p["d"], q, s["w"], s["offsets"], p["y"], a_scale=scale, b_scale=s["t"], bias=s["bias"], **p["ws"])
        return p["y"]
    h.gemm_grouped(p["d"], s["x"], s["w"], s["offsets"], p["y"], bias=s["bias"], **p["ws"])
    if not case["train"]:
        return p["y"]
    h.gemm_grouped_dx(p["d_dx"], s["dy"], s["w"], s["offsets"], p["dx"], relu_of=s["x"], **p["ws"])
    h.gemm_grouped_dw(p["d_dw"], s["x"], s["dy"], s["offsets"], p["dw"], dbias=p["db"], **p["ws"])
    return p["y"], p["dx"], p["dw"], p["db"]


def _quantize(x):
    """Rows to 8 bits in elementary operations: q and the scales."""
    v = x.float()
    top = v.abs().amax(1)
    # the scale's upper 16 significant bits, rounded up
    s = (((top / 127).view(torch.int32) + 0xff) & ~0xff).view(torch.float32).clamp_(min=2.0 ** -126)
    c = s[:, None]
    q = (v / c).round_()
    # v - q * c is exact: one step back where the quotient was rounded onto or over a tie, and ties go to even numbers
    rest = v - q * c
    half = 0.5 * c
    odd = (q - 2 * (0.5 * q).floor()) == 1
    up = (rest > half) | ((rest == half) & odd)
    down = (rest < -half) | ((rest == -half) & odd)
    q = q + up.float() - down.float()
    return q.to(torch.int8), s


def _finish(y, bias, relu, dtype):
    if bias is not None:
        y = y + bias
    if relu:
        y = torch.where(y < 0, torch.zeros_like(y), y)
    return y.to(dtype)


def _run_plain(state):
    case, s = state["case"], state["inputs"]
    if case["kind"] == "quantize":
        q, scale = _quantize(s["x"])
        return q.float() * scale[:, None], scale
    q, scale, bias = s.get("q"), s.get("s"), s["bias"]
    if case["quantize"]:
        q, scale = _quantize(s["x"])
    if case["kind"] == "product8":
        y = torch.matmul(q.float(), s["w"].float().t()) * scale[:, None] * s["t"]
        return _finish(y, bias, case["relu"], _TYPES[case["out"]][0])
    at, groups = s["at"], case["groups"]
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    y = torch.empty(case["rows"], case["N"], dtype=dtype, device="cuda")
    if case["train"]:
        dx = torch.empty(case["rows"], case["K"], dtype=dtype, device="cuda")
        dw = torch.zeros(groups, case["N"], case["K"], device="cuda")
        db = torch.zeros(groups, case["N"], device="cuda")
    for e in range(groups):
        lo, hi = at[e], at[e + 1]
        if lo == hi:
            continue
        w = s["w"][e].float()
        b = bias[e] if bias is not None else None
        if case["dtype"] == "i8":
            part = torch.matmul(q[lo:hi].float(), w.t()) * scale[lo:hi, None] * s["t"][e]
        else:
            x = s["x"][lo:hi].float()
            part = torch.matmul(x, w.t())
        y[lo:hi] = _finish(part, b, case["relu"], dtype)
        if case["train"]:
            dy = s["dy"][lo:hi].float()
            dx[lo:hi] = (torch.matmul(dy, w) * (x > 0)).to(dtype)
            dw[e] = torch.matmul(dy.t(), x)
            db[e] = dy.sum(0)
    return (y, dx, dw, db) if case["train"] else y


# ---- the definition, in 64 bits -------------------------------------------------------------------------------------------

def _exact_rows(x):
    """(q, s) of the definition: the quotient of 64-bit numbers is exact enough to tell every tie of 24-bit by 16-bit values."""
    x = x.double()
    mantissa, power = torch.frexp((x.abs().amax(dim=1) / 127.0).float().double())
    s = torch.ldexp(torch.ceil(mantissa * 65536.0) / 65536.0, power).clamp(min=2.0 ** -126)
    return torch.round(x / s.unsqueeze(1)), s


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "quantize":
        q, scale = _exact_rows(s["x"])
        return q * scale.unsqueeze(1), scale
    if case["kind"] == "product8" or case["dtype"] == "i8":
        if case["quantize"]:
            q, scale = _exact_rows(s["x"])
        else:
            q, scale = s["q"].double(), s["s"].double()
        a = q * scale.unsqueeze(1)
        del q
    else:
        a = s["x"].double()
    spans = [(0, 0, a.shape[0])] if case["kind"] == "product8" else [(e, s["at"][e], s["at"][e + 1]) for e in range(case["groups"])]
    y = torch.zeros(a.shape[0], case["N"], dtype=torch.float64, device="cuda")
    grads = None
    if case.get("train"):
        grads = (torch.zeros_like(a), torch.zeros(s["w"].shape, dtype=torch.float64, device="cuda"),
                 torch.zeros(case["groups"], case["N"], dtype=torch.float64, device="cuda"))
    w_all, bias = s["w"].view(-1, case["N"], case["K"]), s["bias"]
    for e, lo, hi in spans:
        if hi <= lo:
            continue
        b = w_all[e].double()
        if "t" in s:
            b = b * s["t"].view(-1, case["N"])[e].double().unsqueeze(1)
        out = a[lo:hi] @ b.T
        if bias is not None:
            out += bias.view(-1, case["N"])[e].double()
        y[lo:hi] = out.clamp(min=0.0) if case["relu"] else out
        if grads is not None:
            g = s["dy"][lo:hi].double()
            grads[0][lo:hi] = torch.where(a[lo:hi] > 0, g @ b, torch.zeros((), dtype=torch.float64, device="cuda"))
            grads[1][e] = g.T @ a[lo:hi]
            grads[2][e] = g.sum(dim=0)
    return (y, *grads) if grads is not None else y
