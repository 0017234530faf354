"""Products with low-rank adapters where values or extents are at an end: infinities in an adapter, and more rows than one launch has workgroups for."""
import numpy as np
import pytest
import torch

import paper_2210_12415_amd as alt
from rows_util import EPS, HALF, f64, matrix, normal, ws

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.fixture(scope="module")
def h():
    return alt.Handle()


# (few rows; the product in fp32 with a last pass; the adapters' part in the product's tiles, of every kind there)
@pytest.mark.parametrize("M,N,K,G,r", [(16, 128, 256, 4, 16), (300, 640, 256, 4, 16), (800, 4096, 512, 64, 4), (700, 1024, 512, 4, 16), (3000, 2048, 256, 4, 16), (3000, 2048, 256, 4, 33),
                                       (2100, 1030, 1031, 4, 16)])
@pytest.mark.parametrize("dtype,out", [(alt.BF16, alt.BF16), (alt.BF16, alt.F32), (alt.F32, alt.F32)])
def test_infinities_in_an_adapter_are_the_definitions(h, M, N, K, G, r, dtype, out):
    """An infinity in b meets the row's inner sum once: an infinity of its sign, NaN where the sum is zero.  Inner sums that 8 bits hold whole (what they leave
    is zero) and others, of both signs, and an adapter whose a is zeros."""
    t = {alt.F32: torch.float32, alt.BF16: torch.bfloat16}[dtype]
    ids = torch.tensor(np.sort(np.random.RandomState(M).randint(-1, G, M)), dtype=torch.int32)
    x, w = matrix(normal(1, M, K), t), matrix(normal(2, N, K, std=K ** -0.5), t)
    a, b = matrix(normal(3, G * r, K, std=K ** -0.5), t).view(G, r, K), matrix(normal(4, G * N, r), t).view(G, N, r)
    x[:, 0] = torch.tensor([2.0, -0.5]).repeat(M)[:M].to(t)                  # (of a row's adapter 2 the inner sums are these)
    a[1], a[2] = 0, 0
    a[2, :, 0] = 1
    b[0, ::5, 3], b[0, 1::7, 0], b[1, ::3, 2], b[2, ::4, 1], b[2, 1::4, 0] = INF, -INF, INF, INF, -INF
    b[0, ::35, 1] = -INF                                   # (beside an infinity of the other sign, or of the same)
    d = alt.adapters_desc(M, N, K, G, r, in_dtype=dtype, out_dtype=out)
    y = torch.empty(M, N, dtype={alt.F32: torch.float32, alt.BF16: torch.bfloat16}[out], device="cuda")
    h.gemm_adapters(d, x, w, ids.cuda(), a, b, y, **ws(h.gemm_adapters_workspace_size(d)))
    torch.cuda.synchronize()
    got, X, W, A, B = f64(y), f64(x), f64(w), f64(a), f64(b)
    seen = set()
    for g in range(-1, G):
        m = np.flatnonzero(ids.numpy() == g)
        want = X[m] @ W.T
        if g >= 0:
            inner = X[m] @ A[g].T
            with np.errstate(invalid="ignore"):
                for q in range(r):
                    want = want + inner[:, q:q + 1] * B[g][None, :, q]
        whole = np.isfinite(want)
        at = got[m]
        assert np.isfinite(at[whole]).all(), g
        assert (np.isnan(want) == np.isnan(at)).all(), g
        assert (at[np.isinf(want)] == want[np.isinf(want)]).all(), g
        seen |= {(g, v) for v, is_ in (("inf", np.isinf(want).any()), ("nan", np.isnan(want).any())) if is_}
    assert {(0, "inf"), (0, "nan"), (1, "nan"), (2, "inf")} <= seen and not any(g in (-1, 3) for g, _ in seen)


@pytest.mark.parametrize("M,N,K,G,r", [((1 << 23) + 5, 8, 8, 3, 512), ((1 << 26) + 7, 8, 8, 32, 64)])
def test_more_rows_than_a_launch_has_workgroups(h, M, N, K, G, r):
    """The inner sums of rank 512 have 32 workgroups for 16 rows, a last pass one for four rows: 2^24 workgroups of 256 threads are more threads than one launch has."""
    torch.manual_seed(1)
    x = torch.randn(M, K, device="cuda").bfloat16()
    w, a, b = torch.randn(N, K, device="cuda").bfloat16(), torch.randn(G, r, K, device="cuda").bfloat16(), torch.randn(G, N, r, device="cuda").bfloat16()
    ids = torch.randint(-1, G, (M,), dtype=torch.int32, device="cuda")
    d = alt.adapters_desc(M, N, K, G, r, out_dtype=alt.F32)
    y = torch.full((M, N), float("nan"), device="cuda")
    need = h.gemm_adapters_workspace_size(d)
    h.gemm_adapters(d, x, w, ids, a, b, y, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), ws_bytes=need)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(y).all())
    step = M // 64
    for lo in list(range(0, M - 600, step)) + [M - 600]:                     # 600 rows of each 64th, and the last
        at = slice(lo, lo + 600)
        xs, of = f64(x[at]), ids[at].cpu().numpy()
        want, size = xs @ f64(w).T, K * EPS * (np.abs(xs) @ np.abs(f64(w)).T)
        for g in range(G):
            m = np.flatnonzero(of == g)
            A, B = f64(a[g]), f64(b[g])
            inner, about = xs[m] @ A.T, np.abs(xs[m]) @ np.abs(A).T
            want[m] += inner @ B.T
            size[m] += ((K + 1) * EPS * about + (2.0 ** -16 + EPS) * np.abs(inner)) @ np.abs(B).T + (2 * r + 3) * EPS * (np.abs(inner) @ np.abs(B).T)
        tol = 1.01 * size + 4 * EPS * np.abs(want) + HALF[alt.F32]
        assert (np.abs(f64(y[at]) - want) <= tol).all(), lo
