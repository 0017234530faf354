"""The calls around the layers' products at their largest: more chunks than one launch counts, more rows than a launch has workgroups, buffers of more than 2^32 bytes.
Results that a row has by itself are compared, bit for bit, with those of calls on a few of the rows, which the other tests hold against the formulas."""
import pytest
import torch

import paper_2210_12415_amd as alt
from rows_util import EPS, close, f64, ws

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    return alt.Handle()


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def filled(rows, cols, dtype=torch.bfloat16):
    """Random rows, made of a block of them that is shifted along for each next block, so that no two rows are alike by their place."""
    block = torch.randn(4099, cols, device="cuda").to(dtype)
    out = torch.empty(rows, cols, dtype=dtype, device="cuda")
    for i, lo in enumerate(range(0, rows, len(block))):
        part = out[lo:lo + len(block)]
        part.copy_(torch.roll(block, i % cols, 1)[:len(part)])
    return out


def places(rows, n=150):
    """First rows of the slices that are looked at: both ends, and between them."""
    return sorted({0, rows - n} | {int(f * (rows - n)) for f in (0.1, 0.25, 0.4999, 0.5, 0.75, 0.97)})


def test_exchange_of_more_chunks_than_a_launch_counts(h):
    """4.2 million rows of 512 chunks are 2^31 of them and some; rows of the experts' order are the tokens', turned by a third of them."""
    T, C, n = (1 << 22) + 77, 4096, 150
    d, few = alt.exchange_desc(T, 1, T, C), alt.exchange_desc(n, 1, n, C)
    x, y = filled(T, C), torch.empty(T, C, dtype=torch.bfloat16, device="cuda")
    turn = T // 3
    rows = ((torch.arange(T, device="cuda") + turn) % T).int().view(T, 1)
    some = torch.arange(n, dtype=torch.int32, device="cuda").view(n, 1)
    h.dispatch_rows(d, x, rows, y)
    for lo in places(T - turn) + [T - turn - 3, T - n]:
        at = rows[lo:lo + n, 0].long()
        assert torch.equal(y[at], x[lo:lo + n])
    w = torch.rand(T, 1, device="cuda") + 0.5
    back = torch.empty(T, C, dtype=torch.bfloat16, device="cuda")
    h.combine_rows(d, y, rows, back, weights=w)
    for lo in places(T):
        want = torch.empty(n, C, dtype=torch.bfloat16, device="cuda")
        h.combine_rows(few, x[lo:lo + n].contiguous(), some, want, weights=w[lo:lo + n].contiguous())
        assert torch.equal(back[lo:lo + n], want)
    dx, dw = back, torch.empty(T, 1, device="cuda")
    h.combine_rows_grad(d, x, y, rows, w, dx, dw)
    for lo in places(T):
        want, sums = torch.empty(n, C, dtype=torch.bfloat16, device="cuda"), torch.empty(n, 1, device="cuda")
        mine = x[lo:lo + n].contiguous()
        h.combine_rows_grad(few, mine, mine, some, w[lo:lo + n].contiguous(), want, sums)
        assert torch.equal(dx[rows[lo:lo + n, 0].long()], want) and torch.equal(dw[lo:lo + n], sums)


@pytest.mark.parametrize("rows,cols", [((1 << 20) + 5, 16385), (600_001, 8192), (4_200_001, 1000)])
def test_norm_of_buffers_past_32_bits(h, rows, cols):
    n, both = 150, dict(in_dtype=alt.BF16, out_dtype=alt.BF16)
    d, few = alt.norm_desc(rows, cols, **both), alt.norm_desc(n, cols, **both)
    x, y = filled(rows, cols), torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    gamma, beta = torch.rand(cols, device="cuda") + 0.5, torch.randn(cols, device="cuda")
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    h.layer_norm(d, x, y, gamma=gamma, beta=beta, mean=mean, rstd=rstd)
    for lo in places(rows):
        want, m, r = torch.empty(n, cols, dtype=torch.bfloat16, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        h.layer_norm(few, x[lo:lo + n].contiguous(), want, gamma=gamma, beta=beta, mean=m, rstd=r)
        assert torch.equal(y[lo:lo + n], want) and torch.equal(mean[lo:lo + n], m) and torch.equal(rstd[lo:lo + n], r)
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    h.layer_norm_grad(d, y, x, mean, rstd, dx, gamma=gamma, dgamma=dgamma, dbeta=dbeta, **ws(h.layer_norm_grad_workspace_size(d)))
    for lo in places(rows):
        want = torch.empty(n, cols, dtype=torch.bfloat16, device="cuda")
        h.layer_norm_grad(few, y[lo:lo + n].contiguous(), x[lo:lo + n].contiguous(), mean[lo:lo + n].contiguous(), rstd[lo:lo + n].contiguous(), want, gamma=gamma)
        assert torch.equal(dx[lo:lo + n], want)
    # the columns' sums, of 64 shares or more, each off by its length in half steps
    sums = torch.zeros(4, cols, dtype=torch.float64, device="cuda")
    for lo in range(0, rows, 16384):
        at = slice(lo, lo + 16384)
        dy = y[at].double()
        t = dy * ((x[at].double() - mean[at].double()[:, None]) * rstd[at].double()[:, None])
        sums += torch.stack([t.sum(0), t.abs().sum(0), dy.sum(0), dy.abs().sum(0)])
    s = f64(sums)
    close(dgamma, s[0], (rows / 64 + 83) * EPS * s[1], "dgamma")
    close(dbeta, s[2], (rows / 64 + 80) * EPS * s[3], "dbeta")


def test_route_of_as_many_tokens_as_there_may_be(h):
    T, E, k = 1 << 25, 8, 2
    l = torch.randn(T, E, device="cuda").bfloat16()
    d = alt.route_desc(T, E, k, dtype=alt.BF16, renormalize=True)
    experts, weights, rows = (torch.empty(T, k, dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.int32))
    offsets = torch.empty(E + 1, dtype=torch.int32, device="cuda")
    need = h.route_workspace_size(d)
    h.route(d, l, experts, weights, rows, offsets, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), ws_bytes=need)
    step = 1 << 22
    for lo in range(0, T, step):
        assert torch.equal(experts[lo:lo + step], l[lo:lo + step].float().argsort(dim=1, descending=True, stable=True)[:, :k].int())
    flat = experts.flatten()
    counts = torch.stack([(flat == e).sum() for e in range(E)]).cpu()
    assert torch.equal(offsets.cpu().long(), torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)]))
    order = torch.empty(T * k, dtype=torch.int32, device="cuda")
    for e in range(E):
        at = (flat == e).nonzero()[:, 0]
        order[at] = torch.arange(len(at), dtype=torch.int32, device="cuda") + int(offsets[e])
    assert torch.equal(rows.flatten(), order)
    n, few = 150, alt.route_desc(150, E, k, dtype=alt.BF16, renormalize=True)
    dw, dl = torch.randn(T, k, device="cuda"), torch.empty_like(l)
    h.route_grad(d, l, experts, dw, dl)
    for lo in places(T):
        want = torch.empty(n, E, dtype=torch.bfloat16, device="cuda")
        h.route_grad(few, l[lo:lo + n].contiguous(), experts[lo:lo + n].contiguous(), dw[lo:lo + n].contiguous(), want)
        assert torch.equal(dl[lo:lo + n], want)


@pytest.mark.parametrize("M,N,K,G,r,way", [(70_003, 32768, 64, 3, 16, "fused"), (40_000, 32768, 64, 64, 4, "few"), (140_000, 16384, 64, 64, 4, "beside")])
def test_adapters_of_results_past_32_bits(h, M, N, K, G, r, way):
    x, w = filled(M, K), (torch.randn(N, K, device="cuda") * K ** -0.5).bfloat16()
    a, b = (torch.randn(G, r, K, device="cuda") * K ** -0.5).bfloat16(), torch.randn(G, N, r, device="cuda").bfloat16()
    ids = (torch.arange(M, device="cuda") // 37 % (G + 1) - 1).int()
    d = alt.adapters_desc(M, N, K, G, r)
    need = h.gemm_adapters_workspace_size(d)
    assert (need > M * N * 4) == (way != "fused")
    y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    h.gemm_adapters(d, x, w, ids, a, b, y, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), ws_bytes=need)
    for lo in places(M, 300):
        at = slice(lo, lo + 300)
        X, of = x[at].double(), ids[at].long()
        want, size = X @ w.double().t(), K * EPS * (X.abs() @ w.double().abs().t())
        for g in range(G):
            m = (of == g).nonzero()[:, 0]
            if not len(m):
                continue
            A, B = a[g].double(), b[g].double().t().contiguous()
            inner, about = X[m] @ A.t(), X[m].abs() @ A.abs().t()
            want[m] += inner @ B
            size[m] += ((K + 1) * EPS * about + (2.0 ** -16 + EPS) * inner.abs()) @ B.abs() + (2 * r + 3) * EPS * (inner.abs() @ B.abs())
        tol = 1.01 * size + 4 * EPS * want.abs() + 2.0 ** -8 * (want.abs() + size) + 2.0 ** -132
        assert bool(((y[at].double() - want).abs() <= tol).all()), lo
