"""The choice of experts, their order and its gradient against the definition in 64 bits.

Which experts are chosen and the order of their rows have one right answer.  Weights: exp(x) in fp32 of an x that is itself rounded is off by
(|x| + 2) * 2^-24 of itself, a sum of E scores by (E / 16 + 16) * 2^-24 (16 lanes at least share a row), and a handful of single roundings; a sigmoid by
(|l| + 8) * 2^-24.  Gradients: the same for each score, times the largest of the terms that are subtracted."""
import numpy as np
import pytest
import torch

import paper_2210_12415_amd as alt
from rows_util import EPS, HALF, TINY, TORCH, Guarded, close, equal, f64, matrix, normal, replayed, ws

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.fixture(scope="module")
def h():
    return alt.Handle()


def scores(l, softmax):
    if not softmax:
        with np.errstate(over="ignore"):
            return 1 / (1 + np.exp(-l))
    top = l.max(1, keepdims=True)
    with np.errstate(invalid="ignore"):
        e = np.where(l == -INF, 0.0, np.exp(l - np.where(np.isfinite(top), top, 0.0)))
    return e / np.where(e.sum(1, keepdims=True) > 0, e.sum(1, keepdims=True), 1)


def routed(l, d, bias=None):
    """experts, weights, rows, offsets, and how far weights may be off."""
    l = f64(l)
    T, E = l.shape
    softmax, k = d.score == alt.SCORE_SOFTMAX, d.top_k
    lost = np.isnan(l).any(1) | (softmax & (l == INF).any(1))
    l = np.where(lost[:, None], -INF, l)
    s = scores(l, softmax)
    worth = s if bias is None else s + f64(bias)
    worth = np.where((l == -INF) | np.isnan(worth), -INF, worth)
    key = np.where(worth == -INF, -INF, l if bias is None else worth)
    if d.top_groups < d.groups:
        best = -np.sort(-worth.reshape(T, d.groups, -1), axis=2)[:, :, :d.group_best]
        value = np.where(best[:, :, 0] == -INF, -INF, np.where(best == -INF, 0, best).sum(2))
        place = np.argsort(np.argsort(-value, axis=1, kind="stable"), axis=1, kind="stable")
        key = np.where(np.repeat(place >= d.top_groups, E // d.groups, axis=1), -INF, key)
    order = np.argsort(-key, axis=1, kind="stable")[:, :k]
    none = np.take_along_axis(key, order, 1) == -INF
    experts = np.where(none, -1, order)
    raw = np.where(none, 0, np.take_along_axis(s, order, 1))
    total = raw.sum(1, keepdims=True)
    w = d.scale * (raw / np.where(total > 0, total, 1) if d.renormalize else raw)
    x = np.take_along_axis(l, order, 1)
    with np.errstate(invalid="ignore"):
        reach = np.where(none, 0, np.abs(x - l.max(1, keepdims=True)) if softmax else np.abs(x))
    tol = np.abs(w) * EPS * (reach + reach.max(1, keepdims=True, initial=0) + E / 16 + 40) + TINY[alt.F32]
    w[lost] = np.nan
    flat = experts.reshape(-1)
    rows = np.full(T * k, -1)
    there = np.flatnonzero(flat >= 0)
    rows[there[np.argsort(flat[there], kind="stable")]] = np.arange(len(there))
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[there], minlength=E))])
    return experts, w, rows.reshape(T, k), offsets, tol


def run(h, l, d, bias=None, space=None):
    T, k = d.tokens, d.top_k
    out = [Guarded(T, k, torch.int32), Guarded(T, k, torch.float32), Guarded(T, k, torch.int32), Guarded(1, d.experts + 1, torch.int32)]
    h.route(d, l, *out, bias=bias, **(space or ws(h.route_workspace_size(d), 3)))
    torch.cuda.synchronize()
    assert all(o.untouched() for o in out)
    return [o.t for o in out[:3]] + [out[3].t[0]]


def check(h, l, d, bias=None):
    got, want = run(h, l, d, bias), routed(l, d, bias)
    equal(got[0], want[0], "experts")
    close(got[1], want[1], want[4], "weights")
    equal(got[2], want[2], "rows")
    equal(got[3], want[3], "offsets")
    return got


def logits(T, E, seed=0, masked=0.0, padded=0.0, spread=1.0):
    l = normal(seed + T * 13 + E, T, E, std=spread) + normal(seed + E, E, std=0.5)
    g = torch.Generator().manual_seed(seed + 5)
    if masked:
        l[torch.rand(T, E, generator=g) < masked] = -INF
    if padded:
        l[torch.rand(T, generator=g) < padded] = -INF
    return l


SIZES = [(1, 1, 1), (1, 8, 2), (3, 5, 5), (16, 64, 2), (63, 61, 3), (64, 7, 1), (65, 65, 4), (257, 100, 6), (1000, 128, 8), (33, 129, 2), (300, 256, 8), (5, 1000, 32), (70, 1024, 7), (2049, 16, 2),
         (5003, 61, 3), (20000, 32, 4)]


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("score", [alt.SCORE_SOFTMAX, alt.SCORE_SIGMOID])
@pytest.mark.parametrize("dtype", [alt.F32, alt.BF16])
def test_route(h, T, E, k, score, dtype):
    l = matrix(logits(T, E), TORCH[dtype])
    for renorm, bias in ((False, None), (True, None), (True, normal(E, E, std=0.05).cuda())):
        check(h, l, alt.route_desc(T, E, k, dtype=dtype, score=score, renormalize=renorm, scale=2.5), bias)


@pytest.mark.parametrize("E,groups,top_groups,k", [(64, 8, 4, 6), (256, 8, 4, 8), (256, 4, 1, 8), (96, 3, 2, 5), (60, 60, 7, 4), (1024, 512, 9, 16), (40, 8, 8, 3), (6, 2, 1, 3)])
@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("score", [alt.SCORE_SOFTMAX, alt.SCORE_SIGMOID])
def test_route_by_groups(h, E, groups, top_groups, k, best, score):
    l = matrix(logits(333, E, 3, masked=0.15), torch.float32)
    for bias in (None, normal(E, E, std=0.1).cuda()):
        check(h, l, alt.route_desc(333, E, k, score=score, groups=groups, top_groups=top_groups, group_best=best, renormalize=True), bias)


@pytest.mark.parametrize("dtype", [alt.F32, alt.BF16])
@pytest.mark.parametrize("score", [alt.SCORE_SOFTMAX, alt.SCORE_SIGMOID])
def test_route_masks_padding_and_special_values(h, dtype, score):
    T, E = 500, 60
    l = logits(T, E, 1, masked=0.9, padded=0.3)
    l[3], l[4], l[5] = -INF, torch.finfo(torch.bfloat16).min, torch.finfo(torch.bfloat16).max
    l[6, 7] = float("nan")
    l[7, 9] = INF
    l[8] = float("nan")
    l[9], l[9, 59] = -INF, 0.5
    l[10, :] = -90.0
    l[11] = -INF
    l[11, 5], l[11, 6] = float("nan"), -INF
    l = matrix(l, TORCH[dtype])
    for renorm in (False, True):
        check(h, l, alt.route_desc(T, E, 4, dtype=dtype, score=score, renormalize=renorm))
        check(h, l, alt.route_desc(T, E, 4, dtype=dtype, score=score, groups=12, top_groups=5, renormalize=renorm))


def test_route_ties_go_to_the_lower_index(h):
    T, E = 200, 96
    g = torch.Generator().manual_seed(1)
    l = torch.randint(0, 3, (T, E), generator=g).float()
    for score in (alt.SCORE_SOFTMAX, alt.SCORE_SIGMOID):
        for bias in (None, (torch.randint(0, 2, (E,), generator=g).float()).cuda()):
            check(h, matrix(l, torch.float32), alt.route_desc(T, E, 9, score=score, renormalize=True), bias)
            check(h, matrix(l, torch.float32), alt.route_desc(T, E, 9, score=score, groups=8, top_groups=3), bias)


def test_route_compares_choices_beyond_32_bits(h):
    """Choices that 24 bits do not tell apart: scores that differ by parts in 2^40 over a bias of one, both ways."""
    T, E = 64, 64
    l = normal(2, T, E, std=2.0 ** -18) - 12
    l = matrix(l, torch.float32)
    for score in (alt.SCORE_SOFTMAX, alt.SCORE_SIGMOID):
        for bias in (torch.ones(E), torch.linspace(0, 2.0 ** -30, E), torch.where(torch.arange(E) % 2 == 0, 1.0, -1.0)):
            check(h, l, alt.route_desc(T, E, 8, score=score), bias.cuda())
            check(h, l, alt.route_desc(T, E, 4, score=score, groups=8, top_groups=2), bias.cuda())
    # saturated sigmoids: logits still order them where there is no bias
    big = matrix(normal(3, T, E, std=3.0) + 60, torch.float32)
    check(h, big, alt.route_desc(T, E, 8, score=alt.SCORE_SIGMOID, renormalize=True))


@pytest.mark.parametrize("E,k", [(8, 5), (64, 8), (200, 7), (256, 9), (257, 6), (300, 17), (512, 8), (512, 20), (1024, 8), (1000, 31), (256, 32)])
def test_route_orders_of_every_shape(h, E, k):
    """Equal logits, both zeros, all negative, few left, near each other and, by the bias, more of them near the last choice than a row has lanes."""
    T = 150
    g = torch.Generator().manual_seed(E + k)
    steps = torch.randint(-3, 3, (T, E), generator=g).float()
    signs = torch.where(torch.rand(T, E, generator=g) < 0.5, -0.0, 0.0)
    few = logits(T, E, 3, masked=0.9)
    near = normal(5, T, E, std=2.0 ** -18) - 12
    largest = torch.where(torch.rand(T, E, generator=g) < 0.1, torch.finfo(torch.float32).max, 0.0)
    largest[torch.rand(T, E, generator=g) < 0.02] = INF
    for l in (steps, signs, steps - 8, few, near, -largest, logits(T, E, 9)):
        l = matrix(l, torch.float32)
        for bias in (None, torch.linspace(0, 2.0 ** -30, E).cuda(), normal(3, E, std=0.1).cuda()):
            check(h, l, alt.route_desc(T, E, k, score=alt.SCORE_SIGMOID, renormalize=True), bias)
            check(h, l, alt.route_desc(T, E, k, score=alt.SCORE_SOFTMAX), bias)
    check(h, matrix(largest, torch.float32), alt.route_desc(T, E, k, score=alt.SCORE_SIGMOID))


@pytest.mark.parametrize("E,groups,top_groups,k", [(512, 8, 4, 8), (512, 64, 20, 12), (300, 10, 3, 8), (300, 3, 2, 20)])
def test_route_by_groups_of_more_experts(h, E, groups, top_groups, k):
    for l in (logits(333, E, 3, masked=0.15), normal(5, 333, E, std=2.0 ** -18) - 12):
        l = matrix(l, torch.float32)
        for bias in (None, normal(E, E, std=0.1).cuda(), torch.ones(E).cuda()):
            for best in (1, 2):
                check(h, l, alt.route_desc(333, E, k, score=alt.SCORE_SIGMOID, groups=groups, top_groups=top_groups, group_best=best, renormalize=True), bias)


def test_route_biases_that_bar_or_force(h):
    T, E = 100, 40
    l = matrix(logits(T, E, 7), torch.float32)
    bias = normal(8, E, std=0.1)
    bias[3], bias[4], bias[5], bias[6] = -INF, float("nan"), INF, INF
    for groups, top_groups in ((1, 1), (8, 2)):
        got = check(h, l, alt.route_desc(T, E, 3, score=alt.SCORE_SIGMOID, groups=groups, top_groups=top_groups, renormalize=True), bias.cuda())
        assert not ((got[0] == 3) | (got[0] == 4)).any() and (got[0][:, 0] == 5).all()
    everyone = torch.full((E,), -INF)
    got = check(h, l, alt.route_desc(T, E, 3, score=alt.SCORE_SIGMOID, renormalize=True), everyone.cuda())
    assert (got[0] == -1).all() and not got[1].any() and not got[3].any()


def test_route_renormalizes_scores_that_are_lost_beside_the_largest(h):
    """Softmax scores of e^-120 and less of which a bias makes the choice: their shares are still right."""
    l = torch.full((4, 16), -30.0)
    l[:, 0] = 100.0
    l[:, 3], l[:, 5] = -20.0, -21.0
    bias = torch.zeros(16)
    bias[[3, 5]] = 10.0
    bias[0] = -10.0
    check(h, matrix(l, torch.float32), alt.route_desc(4, 16, 2, renormalize=True), bias.cuda())


def test_route_one_expert_takes_all_and_strides(h):
    T, E = 3000, 24
    l = logits(T, E, 2)
    l[:, 17] += 100
    check(h, matrix(l, torch.bfloat16, 31, 1), alt.route_desc(T, E, 1, dtype=alt.BF16, stride=31))
    check(h, matrix(l, torch.float32, 25, 1), alt.route_desc(T, E, 24, stride=25))


def test_route_without_tokens(h):
    d = alt.route_desc(0, 30, 2)
    offsets = torch.full((31,), 9, dtype=torch.int32, device="cuda")
    h.route(d, None, None, None, None, offsets, **ws(h.route_workspace_size(d)))
    assert not offsets.any()
    h.route_grad(d, None, None, None, None)


@pytest.mark.parametrize("T,E,k", [(4096, 256, 2), (4097, 256, 2), (16384, 64, 1), (16385, 64, 1), (9000, 1000, 3), (3000, 300, 20)])
def test_route_ranks_of_few_and_many_workgroups(h, T, E, k):
    check(h, matrix(logits(T, E, 2, masked=0.2, padded=0.1), torch.bfloat16), alt.route_desc(T, E, k, dtype=alt.BF16))


def test_route_many_tokens(h):
    T, E, k = (1 << 20) + 333, 8, 2
    l = torch.randn(T, E, device="cuda")
    d = alt.route_desc(T, E, k)
    experts, weights, rows, offsets = run(h, l, d)
    best = l.argsort(dim=1, descending=True, stable=True)[:, :k].int()
    assert torch.equal(experts, best)
    flat = best.flatten().long()
    want = torch.empty(T * k, dtype=torch.int32, device="cuda")
    want[torch.sort(flat, stable=True)[1]] = torch.arange(T * k, dtype=torch.int32, device="cuda")
    assert torch.equal(rows.flatten(), want)
    assert torch.equal(offsets.cpu(), torch.cat([torch.zeros(1), torch.bincount(flat.cpu(), minlength=E).cumsum(0)]).int())


def gradient(l, d, experts, dw):
    """dlogits and how far they may be off."""
    l, dw = f64(l), f64(dw)
    T, E = l.shape
    softmax = d.score == alt.SCORE_SOFTMAX
    s = scores(l, softmax)
    chosen = (experts >= 0) & (experts < E)
    at = np.where(chosen, experts, 0)
    raw = np.where(chosen, np.take_along_axis(s, at, 1), 0)
    dw = np.where(chosen, dw, 0)
    total = raw.sum(1, keepdims=True)
    total = np.where(total > 0, total, 1)
    if d.renormalize:
        ds, e_ds = d.scale / total * (dw - (dw * raw).sum(1, keepdims=True) / total), d.scale / total * (np.abs(dw) + (np.abs(dw) * raw).sum(1, keepdims=True) / total)
    else:
        ds, e_ds = d.scale * dw, d.scale * np.abs(dw)
    full, size = np.zeros((T, E)), np.zeros((T, E))
    for j in range(experts.shape[1]):
        np.add.at(full, (np.arange(T), at[:, j]), np.where(chosen[:, j], ds[:, j], 0))
        np.add.at(size, (np.arange(T), at[:, j]), np.where(chosen[:, j], e_ds[:, j], 0))
    with np.errstate(invalid="ignore"):
        top = l.max(1, keepdims=True)
        reach = np.where(l == -INF, 0, np.abs(l - top) if softmax else np.abs(l))
    reach = reach + np.where(chosen, np.take_along_axis(reach, at, 1), 0).max(1, keepdims=True)
    C = EPS * (2 * reach + E / 16 + 64)
    if softmax:
        dl, tol = s * (full - (ds * raw).sum(1, keepdims=True)), C * s * (size + (e_ds * raw).sum(1, keepdims=True))
    else:
        rest = scores(-np.where(np.isfinite(l), l, -1e4), False)
        dl, tol = full * s * rest, C * size * s * rest
    dl = np.where(chosen.any(1)[:, None], dl, 0)
    return dl, tol + HALF[d.dtype] * (np.abs(dl) + tol) + TINY[d.dtype]


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("score", [alt.SCORE_SOFTMAX, alt.SCORE_SIGMOID])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("dtype", [alt.F32, alt.BF16])
def test_route_gradient(h, T, E, k, score, renorm, dtype):
    l = matrix(logits(T, E, 11, masked=0.1, padded=0.1), TORCH[dtype], E + 3, 1)
    d = alt.route_desc(T, E, k, dtype=dtype, score=score, renormalize=renorm, scale=1.5, stride=E + 3)
    experts = run(h, l, d)[0]
    dw = normal(T + E, T, k).cuda()
    dw[experts < 0] = float("nan")                       # of no choice: not looked at
    out = Guarded(T, E, TORCH[dtype], E + 3, 1)
    h.route_grad(d, l, experts, dw, out)
    torch.cuda.synchronize()
    assert out.untouched()
    want, tol = gradient(l, d, experts.cpu().numpy(), torch.nan_to_num(dw))
    close(out.t, want, tol, "dlogits")


@pytest.mark.parametrize("score", [alt.SCORE_SOFTMAX, alt.SCORE_SIGMOID])
@pytest.mark.parametrize("renorm", [False, True])
def test_route_gradient_against_differences(h, score, renorm):
    T, E, k = 40, 24, 4
    l = logits(T, E, 3)
    d = alt.route_desc(T, E, k, score=score, renormalize=renorm, scale=0.7)
    bias = normal(4, E, std=0.02).cuda()
    experts = run(h, matrix(l, torch.float32), d, bias)[0]
    dw, out = normal(9, T, k), torch.empty(T, E, device="cuda")
    h.route_grad(d, matrix(l, torch.float32), experts, dw.cuda(), out)
    e = experts.cpu().numpy()

    def weights(l):
        raw = np.take_along_axis(scores(l, score == alt.SCORE_SOFTMAX), e, 1)
        return 0.7 * (raw / raw.sum(1, keepdims=True) if renorm else raw)
    way, step = np.random.RandomState(0).standard_normal((T, E)), 1e-5
    slope = ((weights(f64(l) + step * way) - weights(f64(l) - step * way)) * f64(dw)).sum(1) / (2 * step)
    got = (f64(out) * way).sum(1)
    assert np.abs(slope - got).max() <= 1e-5 * max(1.0, np.abs(f64(out) * way).sum(1).max())


def test_route_gradient_of_renormalized_scores_beside_a_larger_one(h):
    l = torch.full((4, 16), -30.0)
    l[:, 0], l[:, 3], l[:, 5] = 100.0, -20.0, -21.0
    l = matrix(l, torch.float32)
    d = alt.route_desc(4, 16, 2, renormalize=True)
    experts, dw, out = torch.tensor([[3, 5]] * 4, dtype=torch.int32, device="cuda"), normal(1, 4, 2).cuda(), torch.empty(4, 16, device="cuda")
    h.route_grad(d, l, experts, dw, out)
    want, tol = gradient(l, d, experts.cpu().numpy(), dw)
    close(out, want, tol)
    assert out[:, 3].abs().min() > 0


def test_route_gradient_same_expert_twice_and_none(h):
    """Choices of the caller's own: an expert that stands twice gets both parts, numbers outside the experts have none."""
    T, E = 30, 12
    l = matrix(logits(T, E, 4), torch.float32)
    for score in (alt.SCORE_SOFTMAX, alt.SCORE_SIGMOID):
        d = alt.route_desc(T, E, 3, score=score)
        experts = torch.tensor([[2, 2, 5], [-1, 12, 0], [-1, -1, 99]] * 10, dtype=torch.int32, device="cuda")
        dw, out = normal(6, T, 3).cuda(), torch.empty(T, E, device="cuda")
        h.route_grad(d, l, experts, dw, out)
        want, tol = gradient(l, d, experts.cpu().numpy(), dw)
        close(out, want, tol)
        assert not out[2::3].any()


@pytest.mark.parametrize("T", [16, 3000])
def test_route_captured_on_another_stream_and_replayed(h, T):
    E, k = 64, 4
    l = matrix(logits(T, E, 1, masked=0.1, padded=0.2), torch.bfloat16)
    d = alt.route_desc(T, E, k, dtype=alt.BF16, renormalize=True)
    outs = [torch.empty(T, k, dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.int32)] + [torch.empty(E + 1, dtype=torch.int32, device="cuda"), torch.empty_like(l)]
    dw, space = normal(2, T, k).cuda(), ws(h.route_workspace_size(d))

    def once():
        h.route(d, l, *outs[:4], **space)
        h.route_grad(d, l, outs[0], dw, outs[4])
    replayed(once, outs, lambda: [o.fill_(3) for o in outs])
