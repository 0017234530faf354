"""Routing where values leave the range of 32 bits, against the definition in 64: renormalized sigmoid weights of logits far below zero, and their gradients;
biases of infinity and of the lowest value by groups.

Shares of the chosen scores are quotients of exponentials: each is off by (|x| + 2) * 2^-24 of itself, x the difference of two logits, which is itself rounded, the sum
of up to 32 of them by 32 * 2^-24 more, and a handful of single roundings."""
import numpy as np
import pytest
import torch

import paper_2210_12415_amd as alt
from rows_util import EPS, HALF, TINY, TORCH, close, equal, f64, matrix, normal, ws

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.fixture(scope="module")
def h():
    return alt.Handle()


def run(h, l, d, bias=None):
    outs = [torch.full((d.tokens, d.top_k), 7, dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.int32)] + [torch.empty(d.experts + 1, dtype=torch.int32, device="cuda")]
    h.route(d, l, *outs, bias=bias, **ws(h.route_workspace_size(d)))
    torch.cuda.synchronize()
    return outs


def shares(v):
    """Of rows of chosen logits (-inf: none), sigmoid(v) / sum sigmoid(v), by exp(v - m) / (1 + exp(v)) with the largest of the row, m, or 0: nothing under- or
    overflows."""
    m = np.minimum(v.max(1, keepdims=True), 0)
    m = np.where(np.isfinite(m), m, 0)
    with np.errstate(over="ignore", under="ignore"):
        s = np.where(v < 0, np.exp(np.minimum(v, 0) - m) / (1 + np.exp(np.minimum(v, 0))), np.exp(-m) / (1 + np.exp(-np.maximum(v, 0))))
    total = s.sum(1, keepdims=True)
    return s / np.where(total > 0, total, 1)


LEVELS = [-5, -20, -24, -60, -86, -88, -95, -100, -103, -104, -120, -300, -700, -740]


def far(T, E, level, dtype, seed):
    """Logits of `level` give or take a few, a fifth of them masked; a row beside an expert of another size, one with a single expert, one without."""
    l = normal(seed + int(-level), T, E, std=1.5) + level
    l[torch.rand(T, E, generator=torch.Generator().manual_seed(seed)) < 0.2] = -INF
    l[1], l[2] = -INF, -INF
    l[2, E // 2] = level
    l[3, 0], l[4, 1] = level + 20, level - 30
    return matrix(l, TORCH[dtype])


@pytest.mark.parametrize("level", LEVELS)
@pytest.mark.parametrize("dtype", [alt.F32, alt.BF16])
@pytest.mark.parametrize("T,E,k", [(70, 12, 2), (33, 61, 8), (20, 300, 5), (10, 1000, 32), (300, 200, 20)])
def test_renormalized_sigmoid_of_logits_far_below_zero(h, T, E, k, dtype, level):
    l = far(T, E, level, dtype, 1)
    d = alt.route_desc(T, E, k, dtype=dtype, score=alt.SCORE_SIGMOID, renormalize=True, scale=1.5)
    experts, weights = run(h, l, d)[:2]
    full = f64(l)
    order = np.argsort(-full, axis=1, kind="stable")[:, :k]
    v = np.take_along_axis(full, order, 1)
    equal(experts, np.where(v == -INF, -1, order), "experts")
    s = shares(v)
    with np.errstate(invalid="ignore"):
        reach = np.where(v == -INF, 0, np.abs(v - v.max(1, keepdims=True)) + np.minimum(np.abs(v), 100))
    reach = reach + reach.max(1, keepdims=True) + k + 16
    close(weights, 1.5 * s, 1.5 * s * EPS * reach + TINY[alt.F32], "weights")
    # the gradient: share * (dweight - mean) * (1 - sigmoid) * scale
    dw, out = normal(3, T, k), torch.empty(T, E, dtype=TORCH[dtype], device="cuda")
    h.route_grad(d, l, experts, dw.cuda(), out)
    up = np.where(v == -INF, 0, f64(dw))
    mean, size = (s * up).sum(1, keepdims=True), (s * np.abs(up)).sum(1, keepdims=True)
    with np.errstate(over="ignore"):
        rest = 1 / (1 + np.exp(np.where(v == -INF, 0, v)))
    want, tol = np.zeros((T, E)), np.zeros((T, E))
    np.put_along_axis(want, order, np.where(v == -INF, 0, 1.5 * s * (up - mean) * rest), 1)
    np.put_along_axis(tol, order, np.where(v == -INF, 0, 1.5 * s * (np.abs(up) + size) * EPS * (2 * reach + 16)), 1)
    close(out, want, tol + HALF[dtype] * (np.abs(want) + tol) + TINY[dtype], "dlogits")


def test_renormalized_sigmoid_of_two_logits(h):
    """Two logits one apart have the shares 0.7311 and 0.2689 wherever below zero they are; where 64 bits have nothing left of either the sum of zero counts as one."""
    at = torch.tensor([-30.0, -60.0, -87.0, -95.0, -100.0, -102.0, -104.0, -200.0, -700.0, -740.0])
    l = torch.full((len(at) + 1, 4), -INF)
    l[:-1, 1], l[:-1, 2] = at - 1, at
    l[-1, 1], l[-1, 2] = -1001.0, -1000.0
    l = matrix(l, torch.float32)
    d = alt.route_desc(len(at) + 1, 4, 2, score=alt.SCORE_SIGMOID, renormalize=True)
    experts, weights, *_ = run(h, l, d)
    equal(experts, np.array([[2, 1]] * (len(at) + 1)))
    first = 1 / (1 + np.exp(-1.0))
    close(weights, np.array([[first, 1 - first]] * len(at) + [[0.0, 0.0]]), 8 * EPS)
    out = torch.empty(len(at) + 1, 4, device="cuda")
    h.route_grad(d, l, experts, torch.tensor([[2.0, -1.0]] * (len(at) + 1), device="cuda"), out)
    mean = 2 * first - (1 - first)
    close(out, np.array([[0, (1 - first) * (-1 - mean), first * (2 - mean), 0]] * len(at) + [[0.0] * 4]), 32 * EPS)


@pytest.mark.parametrize("score", [alt.SCORE_SOFTMAX, alt.SCORE_SIGMOID])
@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("E,groups,top_groups,k", [(64, 8, 3, 6), (128, 8, 2, 5), (256, 8, 4, 8), (512, 16, 3, 8), (1024, 8, 3, 20), (60, 12, 4, 6), (256, 4, 1, 16)])
def test_biases_of_infinity_by_groups(h, E, groups, top_groups, k, best, score):
    """Experts that a bias of infinity forces, several of them side by side: their groups are worth infinity, ties go to the lower index."""
    T, each = 90, E // groups
    l = normal(E, T, E)
    l[torch.rand(T, E, generator=torch.Generator().manual_seed(E)) < 0.2] = -INF
    bias = normal(7, E, std=0.1)
    last = (groups - 1) * each
    bias[[last, last + 1, last + 2, each, each + 1]] = INF
    bias[2 * each] = INF
    l = matrix(l, torch.float32)
    experts = run(h, l, alt.route_desc(T, E, k, score=score, groups=groups, top_groups=top_groups, group_best=best), bias.cuda())[0]
    full, add = f64(l), f64(bias)
    if score == alt.SCORE_SOFTMAX:
        e = np.exp(full - full.max(1, keepdims=True))
        s = e / e.sum(1, keepdims=True)
    else:
        s = 1 / (1 + np.exp(-full))
    key = np.where(full == -INF, -INF, s + add)
    two = -np.sort(-key.reshape(T, groups, each), axis=2)[:, :, :best]
    worth = np.where(two[:, :, 0] == -INF, -INF, np.where(two == -INF, 0, two).sum(2))
    place = np.argsort(np.argsort(-worth, axis=1, kind="stable"), axis=1, kind="stable")
    key = np.where(np.repeat(place >= top_groups, each, axis=1), -INF, key)
    order = np.argsort(-key, axis=1, kind="stable")[:, :k]
    equal(experts, np.where(np.take_along_axis(key, order, 1) == -INF, -1, order), "experts")


def groups_and_experts(l, bias, groups, top_groups, best, k, softmax):
    """The experts of each token, choices and worths in 64 bits."""
    full, (T, E) = f64(l), l.shape
    with np.errstate(invalid="ignore"):
        e = np.exp(full - np.where(np.isfinite(full.max(1)), full.max(1), 0)[:, None])
    s = e / np.maximum(e.sum(1, keepdims=True), 1e-300) if softmax else 1 / (1 + np.exp(-full))
    key = np.where(full == -INF, -INF, s + f64(bias))
    two = -np.sort(-key.reshape(T, groups, E // groups), axis=2)[:, :, :best]
    worth = np.where(two[:, :, 0] == -INF, -INF, np.where(two == -INF, 0, two).sum(2))
    place = np.argsort(np.argsort(-worth, axis=1, kind="stable"), axis=1, kind="stable")
    key = np.where(np.repeat(place >= top_groups, E // groups, axis=1), -INF, key)
    order = np.argsort(-key, axis=1, kind="stable")[:, :k]
    return np.where(np.take_along_axis(key, order, 1) == -INF, -1, order)


@pytest.mark.parametrize("score", [alt.SCORE_SOFTMAX, alt.SCORE_SIGMOID])
@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("E,groups,top_groups,k", [(64, 8, 4, 20), (256, 8, 4, 16), (60, 12, 5, 9), (512, 16, 5, 32), (1024, 8, 3, 24), (416, 8, 6, 21)])
def test_biases_of_the_lowest_value_by_groups(h, E, groups, top_groups, k, best, score):
    """Experts that a bias of the type's lowest value puts last are still before those that a logit of -inf takes out; so are groups of them, whose worth of two is beyond
    that type."""
    T, each = 120, E // groups
    l = normal(E + 1, T, E)
    for t in range(T):                                     # but for two, all groups are out for some tokens
        l[t, each * (t % 4 + 2):] = -INF
        if t % 5 == 0:
            l[t, :each] = -INF
    low = torch.finfo(torch.float32).min
    for value in (low, 0.9 * low, -low, -0.9 * low):
        bias = normal(7, E, std=0.1)
        bias[each:2 * each] = value
        bias[-each:] = value
        bias[2 * each:2 * each + 2] = value * 0.75
        if groups > 6:
            bias[3 * each:4 * each], bias[4 * each:5 * each] = 0.8 * value, 0.95 * value         # (sums of two that only 64 bits tell apart)
        for logits, add in ((l, bias), (l.flip(1), bias.flip(0))):           # (what is left at either end)
            m = matrix(logits, torch.float32)
            experts = run(h, m, alt.route_desc(T, E, k, score=score, groups=groups, top_groups=top_groups, group_best=best), add.contiguous().cuda())[0]
            equal(experts, groups_and_experts(m, add, groups, top_groups, best, k, score == alt.SCORE_SOFTMAX), "experts")
