"""Rows into the experts' order and back, with the gradients, against the formulas in 64 bits.

Tolerances.  Dispatched rows are copies.  A combined row is a sum of top_k products, each rounded, and one last rounding; dx is a product rounded to fp32
and then to its type; dweights is a sum of `cols` products of which 64 threads at least share the row."""
import numpy as np
import pytest
import torch

import paper_2210_12415_amd as alt
from rows_util import EPS, HALF, TINY, TORCH, Guarded, close, f64, matrix, normal, replayed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    return alt.Handle()


def places(T, k, R, seed=0, gone=0.2):
    """A row for every choice, none twice, some choices and some rows left out."""
    g = torch.Generator().manual_seed(seed + T * 5 + k)
    rows = torch.full((T * k,), -1, dtype=torch.int32)
    n = min(T * k, R)
    rows[torch.randperm(T * k, generator=g)[:n]] = torch.randperm(R, generator=g)[:n].int()
    rows[torch.rand(T * k, generator=g) < gone] = -1
    return rows.view(T, k)


def check(h, T, k, R, C, dtype, lt=0, lr=0, offset=0, rows=None, weights=True):
    d = alt.exchange_desc(T, k, R, C, dtype=dtype, token_stride=lt, row_stride=lr)
    t = TORCH[dtype]
    rows = places(T, k, R) if rows is None else rows
    r, there = rows.numpy(), (rows.numpy() >= 0) & (rows.numpy() < R)
    x, w = matrix(normal(C, T, C), t, lt, offset), normal(T + 1, T, k)
    ye = matrix(normal(C + 1, R, C), t, lr, offset)
    wd = w.cuda() if weights else None
    wn = f64(w) if weights else np.ones((T, k))
    rd = rows.cuda()
    # dispatch
    xe = Guarded(R, C, t, lr, offset)
    h.dispatch_rows(d, x, rd, xe)
    want = np.full((R, C), 77.0)
    token, choice = np.nonzero(there)
    want[r[token, choice]] = f64(x)[token]
    torch.cuda.synchronize()
    assert xe.untouched() and np.array_equal(f64(xe.t), want)
    # combine
    out = Guarded(T, C, t, lt, offset)
    h.combine_rows(d, ye, rd, out, weights=wd)
    picked = np.where(there[:, :, None], f64(ye)[np.where(there, r, 0)], 0)
    terms = wn[:, :, None] * picked
    size, want = np.abs(terms).sum(1), terms.sum(1)
    torch.cuda.synchronize()
    assert out.untouched()
    close(out.t, want, (k + 1) * EPS * size + HALF[dtype] * (np.abs(want) + (k + 1) * EPS * size) + TINY[dtype], "combine")
    # its gradients
    dy = matrix(normal(C + 2, T, C), t, lt, offset)
    dx, dw = Guarded(R, C, t, lr, offset), Guarded(T, k, torch.float32)
    h.combine_rows_grad(d, dy, ye, rd, wd, dx, dw)
    torch.cuda.synchronize()
    assert dx.untouched() and dw.untouched()
    want = np.full((R, C), 77.0)
    want[r[token, choice]] = wn[token, choice][:, None] * f64(dy)[token]
    named = np.zeros(R, dtype=bool)
    named[r[token, choice]] = True
    close(dx.t, want, np.where(named[:, None], (EPS + HALF[dtype]) * 1.01 * np.abs(want) + TINY[dtype], 0), "dx")
    terms = f64(dy)[:, None, :] * picked
    close(dw.t, terms.sum(2), (C / 64 + 16) * EPS * np.abs(terms).sum(2), "dweights")
    # without the weights' gradient
    again = Guarded(R, C, t, lr, offset)
    h.combine_rows_grad(d, dy, None, rd, wd, again, None)
    assert torch.equal(again.t, dx.t)


SIZES = [(1, 1, 1, 1), (1, 2, 2, 7), (3, 2, 9, 8), (16, 2, 32, 2048), (5, 4, 11, 63), (100, 3, 300, 515), (33, 8, 264, 1000), (700, 2, 1400, 768), (9, 1, 9, 4099), (4, 32, 128, 8192), (7, 5, 35, 20011),
         (3000, 2, 6000, 64), (2, 2, 4, 70001)]


@pytest.mark.parametrize("T,k,R,C", SIZES)
@pytest.mark.parametrize("dtype", [alt.F32, alt.BF16])
def test_exchange(h, T, k, R, C, dtype):
    check(h, T, k, R, C, dtype)
    check(h, T, k, R, C, dtype, weights=False)


@pytest.mark.parametrize("dtype", [alt.F32, alt.BF16])
@pytest.mark.parametrize("T,k,R,C,lt,lr", [(50, 3, 170, 63, 65, 71), (40, 2, 80, 512, 513, 515), (40, 2, 90, 1024, 1032, 1028)])
def test_exchange_strides_and_alignment(h, T, k, R, C, lt, lr, dtype):
    check(h, T, k, R, C, dtype, lt, lr, 1)


def test_exchange_rows_outside_are_none(h):
    rows = torch.tensor([[0, 5], [-1, 6], [7, -2147483648], [2147483647, 3], [-5, -1], [4, 1]], dtype=torch.int32)
    check(h, 6, 2, 6, 100, alt.BF16, rows=rows)
    check(h, 6, 2, 6, 100, alt.F32, rows=torch.full((6, 2), -1, dtype=torch.int32))


def test_exchange_choices_without_rows_are_zeros_whatever_lies_in_other_rows(h):
    """NaN and infinities of rows that no choice names reach nothing; a weight that is NaN does."""
    T, k, R, C = 5, 2, 10, 300
    rows = torch.tensor([[0, 1], [2, -1], [-1, -1], [-1, -1], [3, 4]], dtype=torch.int32).cuda()
    ye = torch.full((R, C), float("nan"), device="cuda")
    ye[:5] = normal(1, 5, C).cuda()
    w = torch.tensor([[1.0, 2.0], [0.5, 3.0], [0.0, 0.0], [float("nan")] * 2, [1.0, 1.0]], device="cuda")
    d = alt.exchange_desc(T, k, R, C, dtype=alt.F32)
    out, dw, dx = torch.empty(T, C, device="cuda"), torch.empty(T, k, device="cuda"), torch.zeros(R, C, device="cuda")
    h.combine_rows(d, ye, rows, out, weights=w)
    h.combine_rows_grad(d, out, ye, rows, w, dx, dw)
    assert torch.isfinite(out[[0, 1, 2, 4]]).all() and not out[2].any() and torch.isnan(out[3]).all()
    assert torch.isfinite(dw).all() and not dw[2].any() and not dw[3].any() and dw[1, 1] == 0 and torch.isfinite(dx).all()


def test_exchange_without_tokens_or_rows(h):
    h.dispatch_rows(alt.exchange_desc(0, 2, 4, 8), None, None, None)
    h.combine_rows(alt.exchange_desc(0, 2, 4, 8), None, None, None)
    h.combine_rows_grad(alt.exchange_desc(0, 2, 4, 8), None, None, None, None, None, None)
    d = alt.exchange_desc(3, 2, 0, 8)
    rows, y, dw = torch.full((3, 2), -1, dtype=torch.int32, device="cuda"), torch.full((3, 8), 5.0, dtype=torch.bfloat16, device="cuda"), torch.full((3, 2), 5.0, device="cuda")
    h.dispatch_rows(d, y, rows, None)
    h.combine_rows(d, None, rows, y)
    h.combine_rows_grad(d, y, None, rows, None, None, dw)
    assert not y.any() and not dw.any()


def test_exchange_many_tokens(h):
    T, C = (1 << 20) + 100, 8
    d = alt.exchange_desc(T, 1, T, C, dtype=alt.F32)
    rows = torch.randperm(T, device="cuda").int().view(T, 1)
    x, xe, back = torch.randn(T, C, device="cuda"), torch.empty(T, C, device="cuda"), torch.empty(T, C, device="cuda")
    h.dispatch_rows(d, x, rows, xe)
    assert torch.equal(xe[rows[:, 0].long()], x)
    h.combine_rows(d, xe, rows, back)
    assert torch.equal(back, x)
    dx, dw = torch.empty_like(xe), torch.empty(T, 1, device="cuda")
    h.combine_rows_grad(d, x, xe, rows, None, dx, dw)
    assert torch.equal(dx, xe)
    close(dw[:, 0], (f64(x) ** 2).sum(1), 16 * EPS * (f64(x) ** 2).sum(1))


def test_exchange_offsets_past_32_bits(h):
    """Rows of the experts' order that lie more than 2^32 bytes into it."""
    R, stride, C = 9, 300_000_000, 640
    far = torch.zeros((R - 1) * stride + C, dtype=torch.bfloat16, device="cuda")
    v = far.as_strided((R, C), (stride, 1))
    rows = torch.tensor([[8, 0], [7, 3], [1, -1]], dtype=torch.int32, device="cuda")
    d = alt.exchange_desc(3, 2, R, C, row_stride=stride)
    x, out = normal(1, 3, C).bfloat16().cuda(), torch.empty(3, C, dtype=torch.bfloat16, device="cuda")
    h.dispatch_rows(d, x, rows, far)
    assert torch.equal(v[[8, 0, 7, 3, 1]], x[[0, 0, 1, 1, 2]])
    h.combine_rows(d, far, rows, out, weights=torch.full((3, 2), 0.5, device="cuda"))
    assert torch.equal(out[:2], x[:2]) and torch.equal(out[2], x[2] * 0.5)
    h.combine_rows_grad(d, x, far, rows, torch.full((3, 2), 2.0, device="cuda"), far, None)
    assert torch.equal(v[[8, 0, 7, 3, 1]], x[[0, 0, 1, 1, 2]] * 2)


def test_exchange_captured_on_another_stream_and_replayed(h):
    T, k, C = 300, 3, 520
    d = alt.exchange_desc(T, k, T * k, C)
    rows, w = places(T, k, T * k, gone=0).cuda(), normal(3, T, k).cuda()
    x, ye = normal(1, T, C).bfloat16().cuda(), normal(2, T * k, C).bfloat16().cuda()
    outs = [torch.empty_like(ye), torch.empty_like(x), torch.empty_like(ye), torch.empty(T, k, device="cuda"), torch.empty_like(x)]

    def once():
        h.dispatch_rows(d, x, rows, outs[0])
        h.combine_rows(d, ye, rows, outs[1], weights=w)
        h.combine_rows_grad(d, outs[1], ye, rows, w, outs[2], outs[3])
        h.combine_rows(d, outs[2], rows, outs[4])
    replayed(once, outs, lambda: [o.fill_(3) for o in outs])
