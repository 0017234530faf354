"""Layer norm and its gradients against the formulas in 64 bits.

Tolerances.  A sum of n numbers whose longest chain of additions is D is off by D * 2^-24 * sum|.| at most; a row is summed by 64 threads at least, so D <=
n / 64 + 16 with the threads' tree, and the sums over all rows by 64 shares or more that are joined then, D <= rows / 64 + 80.  Every other operation and
the last rounding count half a step of their result."""
import numpy as np
import pytest
import torch

import paper_2210_12415_amd as alt
from rows_util import EPS, HALF, TINY, TORCH, Guarded, close, f64, matrix, normal, replayed, ws

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 7), (3, 8), (2, 63), (5, 64), (16, 768), (7, 1000), (130, 1024), (600, 1024), (3, 2047), (700, 2048), (9, 4096), (513, 4096), (4, 4099), (2, 8192), (300, 8192),
          (5, 8200), (3, 20011), (1000, 33), (4097, 65), (2, 70001)]
TYPES = [(alt.BF16, alt.BF16), (alt.F32, alt.F32), (alt.BF16, alt.F32), (alt.F32, alt.BF16)]


@pytest.fixture(scope="module")
def h():
    return alt.Handle()


def inputs(rows, cols, seed=0):
    x = normal(seed + rows * 31 + cols, rows, cols) * torch.exp(0.5 * normal(seed + cols, cols)) + normal(seed + cols + 1, cols)
    return x, normal(seed + cols + 2, cols, std=0.2, mean=1.0), normal(seed + cols + 3, cols, std=0.1), normal(seed + rows + cols + 4, rows, cols)


def forward(x, gamma, beta, eps, out):
    """y, mean, rstd and how far each may be off."""
    x = f64(x)
    n = x.shape[1]
    D = n / 64 + 16
    mean = x.mean(1, keepdims=True)
    c = x - mean
    var = (c * c).mean(1, keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    e_mean = (D + 1) * EPS * np.abs(x).mean(1, keepdims=True)
    e_c = e_mean + EPS * np.abs(c)
    e_var = 2 * (np.abs(c) * e_c).mean(1, keepdims=True) + (e_c ** 2).mean(1, keepdims=True) + (D + 3) * EPS * var
    with np.errstate(divide="ignore", invalid="ignore"):
        r_rstd = 0.5 * e_var / (var + eps) + (e_var / (var + eps)) ** 2 + 4 * EPS
    g = np.ones(n) if gamma is None else f64(gamma)
    b = np.zeros(n) if beta is None else f64(beta)
    u = c * rstd
    y = u * g + b
    e_y = np.abs(g) * (rstd * e_c * (1 + r_rstd) + np.abs(u) * (r_rstd + 3 * EPS)) + 2 * EPS * (np.abs(u * g) + np.abs(b))
    return (y, mean[:, 0], rstd[:, 0]), (e_y * 1.01 + HALF[out] * (np.abs(y) + e_y) + TINY[out], e_mean[:, 0], (rstd * r_rstd)[:, 0])


def backward(dy, x, mean, rstd, gamma, dtype):
    dy, x, mean, rstd = f64(dy), f64(x), f64(mean)[:, None], f64(rstd)[:, None]
    m, n = x.shape
    D, S = n / 64 + 16, m / 64 + 80
    g = dy * (1 if gamma is None else f64(gamma))
    u = (x - mean) * rstd
    sg, sgu = g.mean(1, keepdims=True), (g * u).mean(1, keepdims=True)
    dx = rstd * (g - sg - u * sgu)
    e_sg, e_sgu = (D + 2) * EPS * np.abs(g).mean(1, keepdims=True), (D + 5) * EPS * np.abs(g * u).mean(1, keepdims=True)
    e_dx = rstd * (e_sg + np.abs(u) * e_sgu + 8 * EPS * (np.abs(g) + np.abs(sg) + np.abs(u * sgu)))
    return ((dx, (dy * u).sum(0), dy.sum(0)),
            (e_dx + HALF[dtype] * (np.abs(dx) + e_dx) + TINY[dtype], (S + 3) * EPS * np.abs(dy * u).sum(0), S * EPS * np.abs(dy).sum(0)))


def run(h, x, gamma, beta, dy, types, eps=1e-5, strides=(0, 0), saved=True, offset=0):
    rows, cols = x.shape
    d = alt.norm_desc(rows, cols, in_dtype=types[0], out_dtype=types[1], eps=eps, x_stride=strides[0], y_stride=strides[1])
    y = Guarded(rows, cols, TORCH[types[1]], strides[1], offset)
    mean, rstd = Guarded(1, rows, torch.float32), Guarded(1, rows, torch.float32)
    h.layer_norm(d, x, y, gamma=gamma, beta=beta, mean=mean if saved else None, rstd=rstd if saved else None)
    torch.cuda.synchronize()
    assert y.untouched() and mean.untouched() and rstd.untouched()
    if dy is None:
        return y.t, mean.t[0], rstd.t[0]
    dx, dgamma, dbeta = Guarded(rows, cols, TORCH[types[0]], strides[0], offset), Guarded(1, cols, torch.float32), Guarded(1, cols, torch.float32)
    h.layer_norm_grad(d, dy, x, mean, rstd, dx, gamma=gamma, dgamma=dgamma, dbeta=dbeta, **ws(h.layer_norm_grad_workspace_size(d), 1))
    torch.cuda.synchronize()
    assert dx.untouched() and dgamma.untouched() and dbeta.untouched()
    return y.t, mean.t[0], rstd.t[0], dx.t, dgamma.t[0], dbeta.t[0]


def check(h, x, gamma, beta, dy, types, **kw):
    got = run(h, x, gamma, beta, dy, types, **kw)
    want, tol = forward(x, gamma, beta, kw.get("eps", 1e-5), types[1])
    for name, a, b, t in zip(("y", "mean", "rstd"), got, want, tol):
        close(a, b, t, name)
    if dy is not None:
        want, tol = backward(dy, x, got[1], got[2], gamma, types[0])
        for name, a, b, t in zip(("dx", "dgamma", "dbeta"), got[3:], want, tol):
            close(a, b, t, name)
    return got


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("types", TYPES)
def test_norm(h, rows, cols, types):
    x, gamma, beta, dy = inputs(rows, cols)
    check(h, matrix(x, TORCH[types[0]]), gamma.cuda(), beta.cuda(), matrix(dy, TORCH[types[1]]), types)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,cols,ldx,ldy", [(5, 63, 65, 71), (300, 1000, 1001, 1003), (40, 4096, 4104, 4100), (9, 8195, 8197, 8201)])
def test_norm_strides_and_alignment(h, rows, cols, ldx, ldy, types):
    x, gamma, beta, dy = inputs(rows, cols, 9)
    check(h, matrix(x, TORCH[types[0]], ldx, 1), gamma.cuda(), beta.cuda(), matrix(dy, TORCH[types[1]], ldy, 1), types, strides=(ldx, ldy), offset=1)


def test_norm_without_gain_offset_or_statistics(h):
    x, gamma, beta, dy = inputs(33, 520, 4)
    x, dy = matrix(x, torch.bfloat16), matrix(dy, torch.bfloat16)
    both = (alt.BF16, alt.BF16)
    check(h, x, None, None, dy, both)
    check(h, x, gamma.cuda(), None, dy, both)
    check(h, x, None, beta.cuda(), dy, both)
    assert torch.equal(run(h, x, gamma.cuda(), beta.cuda(), None, both, saved=False)[0], run(h, x, gamma.cuda(), beta.cuda(), None, both)[0])
    # dx alone, and one of the sums alone
    d = alt.norm_desc(33, 520)
    _, mean, rstd, dx, dgamma, dbeta = run(h, x, gamma.cuda(), beta.cuda(), dy, both)
    for kw in (dict(), dict(dgamma=torch.empty_like(dgamma)), dict(dbeta=torch.empty_like(dbeta))):
        out = torch.empty(33, 520, dtype=torch.bfloat16, device="cuda")
        h.layer_norm_grad(d, dy, x, mean, rstd, out, gamma=gamma.cuda(), **kw, **(ws(h.layer_norm_grad_workspace_size(d)) if kw else {}))
        assert torch.equal(out, dx)
        for name, v in kw.items():
            assert torch.equal(v, dict(dgamma=dgamma, dbeta=dbeta)[name])


def test_norm_far_from_zero_and_constant_rows(h):
    """The mean is taken away before squares are summed: rows around 1000 keep their digits, and constant rows are zeros (rstd = eps^-1/2)."""
    x = normal(1, 64, 1024) + 1000
    x[3], x[5] = 7.0, 0.0
    x, gamma, beta = matrix(x, torch.float32), normal(2, 1024).cuda(), normal(3, 1024).cuda()
    y, mean, rstd, *_ = check(h, x, gamma, beta, matrix(normal(4, 64, 1024), torch.float32), (alt.F32, alt.F32))
    assert torch.equal(y[3], beta) and torch.equal(y[5], beta)
    assert float(mean[3]) == 7.0


def test_norm_special_values_stay_in_their_rows(h):
    x, gamma, beta, dy = inputs(40, 2048, 2)
    both = (alt.BF16, alt.BF16)
    x, dy, gamma, beta = matrix(x, torch.bfloat16), matrix(dy, torch.bfloat16), gamma.cuda(), beta.cuda()
    clean = run(h, x, gamma, beta, dy, both)
    bad = x.clone()
    bad[7, 100], bad[8, 2047], bad[20, 0] = float("nan"), float("inf"), float("-inf")
    got = run(h, bad, gamma, beta, dy, both)
    lost = torch.zeros(40, dtype=torch.bool)
    lost[[7, 8, 20]] = True
    assert torch.isnan(got[0][lost.cuda()].float()).all() and torch.isnan(got[3][lost.cuda()].float()).all()
    for a, b in zip(got[:4], clean[:4]):
        assert torch.equal(a[~lost.cuda()], b[~lost.cuda()])


def test_norm_without_rows(h):
    d = alt.norm_desc(0, 100)
    h.layer_norm(d, None, None)
    dgamma, dbeta = torch.full((100,), 5.0, device="cuda"), torch.full((100,), 5.0, device="cuda")
    h.layer_norm_grad(d, None, None, None, None, None, dgamma=dgamma, dbeta=dbeta, **ws(h.layer_norm_grad_workspace_size(d)))
    assert not dgamma.any() and not dbeta.any()
    h.layer_norm_grad(d, None, None, None, None, None)


def test_norm_gradients_against_differences(h):
    """sum(dy * y) changes by the gradients times a small change of x, gamma and beta (64-bit differences of the definition)."""
    x, gamma, beta, dy = inputs(11, 96, 6)
    got = run(h, matrix(x, torch.float32), gamma.cuda(), beta.cuda(), matrix(dy, torch.float32), (alt.F32, alt.F32))

    def loss(x, gamma, beta):
        c = x - x.mean(1, keepdims=True)
        return float((f64(dy) * (c / np.sqrt((c * c).mean(1, keepdims=True) + 1e-5) * gamma + beta)).sum())
    at, step = [f64(v) for v in (x, gamma, beta)], 1e-5
    for i, grad in enumerate(got[3:]):
        way = np.random.RandomState(i).standard_normal(at[i].shape)
        up, down = ([v + (k == i) * sign * step * way for k, v in enumerate(at)] for sign in (1, -1))
        slope = (loss(*up) - loss(*down)) / (2 * step)
        # (third derivatives times step^2, and the gradients' own rounding)
        assert abs(slope - float((f64(grad) * way).sum())) <= 1e-5 * max(1.0, np.abs(f64(grad) * way).sum())


def test_norm_many_rows(h):
    """More rows than a launch has workgroups."""
    rows = (1 << 20) + 77
    x = torch.randn(rows, 16, device="cuda")
    d = alt.norm_desc(rows, 16, in_dtype=alt.F32, out_dtype=alt.F32)
    y, mean, rstd, dx = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
    dgamma, dbeta = torch.empty(16, device="cuda"), torch.empty(16, device="cuda")
    h.layer_norm(d, x, y, mean=mean, rstd=rstd)
    want, tol = forward(x, None, None, 1e-5, alt.F32)
    for a, b, t in zip((y, mean, rstd), want, tol):
        close(a, b, t)
    h.layer_norm_grad(d, y, x, mean, rstd, dx, dgamma=dgamma, dbeta=dbeta, **ws(h.layer_norm_grad_workspace_size(d)))
    want, tol = backward(y, x, mean, rstd, None, alt.F32)
    for a, b, t in zip((dx, dgamma, dbeta), want, tol):
        close(a, b, t)


def test_norm_offsets_past_32_bits(h):
    """Rows whose distance times their number is more than 2^32 bytes."""
    rows, stride = 5, 600_000_000
    x = torch.zeros((rows - 1) * stride + 512, dtype=torch.bfloat16, device="cuda")
    v = x.as_strided((rows, 512), (stride, 1))
    v.copy_(normal(3, rows, 512).bfloat16())
    d = alt.norm_desc(rows, 512, x_stride=stride)
    y, mean, rstd = torch.empty(rows, 512, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    h.layer_norm(d, x, y, mean=mean, rstd=rstd)
    want, tol = forward(v, None, None, 1e-5, alt.BF16)
    for a, b, t in zip((y, mean, rstd), want, tol):
        close(a, b, t)


def test_norm_captured_on_another_stream_and_replayed(h):
    x, gamma, beta, dy = inputs(700, 1000, 5)
    x, dy, gamma, beta = matrix(x, torch.bfloat16), matrix(dy, torch.bfloat16), gamma.cuda(), beta.cuda()
    d = alt.norm_desc(700, 1000)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd, dgamma, dbeta = torch.empty(700, device="cuda"), torch.empty(700, device="cuda"), torch.empty(1000, device="cuda"), torch.empty(1000, device="cuda")
    space = ws(h.layer_norm_grad_workspace_size(d))
    outs = [y, mean, rstd, dx, dgamma, dbeta]

    def once():
        h.layer_norm(d, x, y, gamma=gamma, beta=beta, mean=mean, rstd=rstd)
        h.layer_norm_grad(d, dy, x, mean, rstd, dx, gamma=gamma, dgamma=dgamma, dbeta=dbeta, **space)
    replayed(once, outs, lambda: [o.fill_(3) for o in outs])


def test_norm_gives_the_same_bits_again(h):
    x, gamma, beta, dy = inputs(3000, 1024, 8)
    x, dy = matrix(x, torch.bfloat16), matrix(dy, torch.bfloat16)
    first = run(h, x, gamma.cuda(), beta.cuda(), dy, (alt.BF16, alt.BF16))
    for _ in range(3):
        for a, b in zip(first, run(h, x, gamma.cuda(), beta.cuda(), dy, (alt.BF16, alt.BF16))):
            assert torch.equal(a, b)
