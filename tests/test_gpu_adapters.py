"""Products with low-rank adapters beside them, against plain sums in 64 bits.

Tolerances.  fp32 sums of n products, in any order: n * 2^-24 * sum |a||b|.  The inner sums are such sums, scaled (one rounding) and kept to half a step of
16 bits of bf16 operands (2^-16); the outer product adds its own sum over the rank, the bias one rounding, the result its last."""
import numpy as np
import pytest
import torch

import paper_2210_12415_amd as alt
from rows_util import EPS, HALF, TINY, TORCH, Guarded, close, f64, matrix, normal, replayed, ws

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    return alt.Handle()


def reference(x, w, adapter, a, b, scale, bias, relu, out):
    x, w, a, b, ids = f64(x), f64(w), f64(a), f64(b), np.asarray(adapter)
    K, r = x.shape[1], b.shape[2]
    y = x @ w.T
    size = K * EPS * (np.abs(x) @ np.abs(w).T)
    for g in np.unique(ids):
        if g < 0 or g >= len(a):
            continue
        m = np.flatnonzero(ids == g)
        s = 1.0 if scale is None else float(scale[g])
        inner, about = s * (x[m] @ a[g].T), abs(s) * (np.abs(x[m]) @ np.abs(a[g]).T)
        y[m] += inner @ b[g].T
        off = (K + 1) * EPS * about + (2.0 ** -16 + EPS) * np.abs(inner)
        size[m] += off @ np.abs(b[g]).T + (2 * r + 3) * EPS * (np.abs(inner) @ np.abs(b[g]).T)
    if bias is not None:
        y = y + f64(bias)
    size = size + 3 * EPS * np.abs(y)
    if relu:
        y = np.maximum(y, 0)
    return y, size * 1.01 + HALF[out] * (np.abs(y) + size) + TINY[out]


def check(h, M, N, K, G, r, adapter, dtype=alt.BF16, out=None, scaled=True, bias=True, relu=False, strides=(0, 0, 0), offset=0):
    out = dtype if out is None else out
    t = TORCH[dtype]
    x, w = matrix(normal(M + K, M, K), t, strides[0], offset), matrix(normal(N + K, N, K, std=K ** -0.5), t, strides[1], offset)
    a, b = matrix(normal(G + K, G * r, K, std=K ** -0.5), t, 0, offset).view(G, r, K), matrix(normal(G + N, G * N, r, std=r ** -0.5), t, 0, offset).view(G, N, r)
    scale = torch.rand(G, generator=torch.Generator().manual_seed(1)) + 0.5 if scaled else None
    add = normal(N, N, std=0.1) if bias else None
    adapter = torch.as_tensor(adapter, dtype=torch.int32)
    d = alt.adapters_desc(M, N, K, G, r, in_dtype=dtype, out_dtype=out, epilogue=alt.EPI_BIAS * bias + alt.EPI_RELU * relu, lda=strides[0], ldb=strides[1], ldc=strides[2])
    y = Guarded(M, N, TORCH[out], strides[2], offset)
    h.gemm_adapters(d, x, w, adapter.cuda(), a, b, y, scale=None if scale is None else scale.cuda(), bias=None if add is None else add.cuda(),
                    **ws(h.gemm_adapters_workspace_size(d), 5))
    torch.cuda.synchronize()
    assert y.untouched()
    want, tol = reference(x, w, adapter, a, b, scale, add, relu, out)
    close(y.t, want, tol, "y")
    return y.t


def requests(M, G, seed=0, lengths=(1, 40)):
    """Rows of requests of uneven lengths, each with an adapter or none."""
    g, rows = np.random.RandomState(seed), []
    while len(rows) < M:
        rows += [g.randint(-1, G)] * g.randint(*lengths)
    return rows[:M]


# one row to the sizes of every kernel behind the call: few rows, odd alignment, tiles of 64, 128 and 256
SIZES = [(1, 1, 1, 1, 1), (1, 64, 64, 3, 16), (2, 65, 16, 2, 3), (16, 256, 1024, 16, 16), (17, 100, 333, 5, 7), (33, 512, 48, 4, 64), (64, 64, 128, 9, 8), (65, 200, 2049, 3, 33), (100, 1000, 15, 7, 5),
         (257, 513, 640, 6, 24), (300, 768, 768, 40, 4), (513, 300, 1031, 5, 130), (700, 1024, 512, 3, 32), (1500, 768, 256, 8, 16), (2048, 1024, 256, 5, 512)]


@pytest.mark.parametrize("M,N,K,G,r", SIZES)
@pytest.mark.parametrize("dtype", [alt.BF16, alt.F32])
def test_adapters(h, M, N, K, G, r, dtype):
    check(h, M, N, K, G, r, requests(M, G), dtype)


@pytest.mark.parametrize("K", [1, 2, 31, 63, 64, 65, 129, 255, 256, 257, 511, 1000, 2047, 4096, 9999])
@pytest.mark.parametrize("M,G,r", [(5, 3, 16), (16, 2, 40), (20, 20, 5), (48, 3, 17), (600, 4, 20)])
@pytest.mark.parametrize("dtype", [alt.BF16, alt.F32])
def test_adapters_of_every_reduction(h, M, G, r, K, dtype):
    """Reductions that end inside the pieces, the steps and the slices that they are cut into."""
    check(h, M, 80, K, G, r, requests(M, G, K), dtype)


@pytest.mark.parametrize("M,N,K", [(40, 3000, 512), (2100, 2048, 512), (5000, 2048, 128)])
@pytest.mark.parametrize("out", [alt.BF16, alt.F32])
def test_adapters_in_large_tiles(h, M, N, K, out):
    check(h, M, N, K, 6, 16, requests(M, 6, 1, (1, 700)), out=out, relu=True)


@pytest.mark.parametrize("dtype", [alt.BF16, alt.F32])
@pytest.mark.parametrize("M", [1, 16, 48, 400])
def test_adapters_of_every_row_its_own_in_any_order(h, M, dtype):
    order = np.random.RandomState(M).permutation(M)
    check(h, M, 192, 320, M, 8, order, dtype)
    check(h, M, 192, 320, 5, 8, np.random.RandomState(1).randint(-1, 5, M), dtype, scaled=False, bias=False)


def test_adapters_of_no_row_and_numbers_outside(h):
    M, N, K, G = 70, 160, 96, 4
    for ids in ([-1] * M, [4] * M, [2147483647, -2147483648] * (M // 2), ([0, 7, -3, 3] * M)[:M]):
        check(h, M, N, K, G, 16, ids)


@pytest.mark.parametrize("dtype", [alt.BF16, alt.F32])
def test_adapters_strides_and_alignment(h, dtype):
    check(h, 75, 130, 200, 4, 12, requests(75, 4), dtype, strides=(203, 201, 131), offset=1)
    check(h, 75, 136, 208, 4, 16, requests(75, 4), dtype, strides=(216, 224, 144))
    check(h, 600, 513, 301, 4, 9, requests(600, 4), dtype, strides=(303, 305, 517), offset=1)


def test_adapters_equal_the_product_where_no_row_has_one(h):
    """Rows without an adapter: exactly the shared projection."""
    M, N, K = 100, 256, 512
    x, w = matrix(normal(1, M, K), torch.bfloat16), matrix(normal(2, N, K, std=0.05), torch.bfloat16)
    a, b = matrix(normal(3, 2 * 8, K), torch.bfloat16).view(2, 8, K), matrix(normal(4, 2 * N, 8), torch.bfloat16).view(2, N, 8)
    y, plain = torch.empty(M, N, device="cuda"), torch.empty(M, N, device="cuda")
    ids = torch.tensor(([-1] * 30 + [1] * 10 + [-1] * 10) * 2, dtype=torch.int32, device="cuda")
    d = alt.adapters_desc(M, N, K, 2, 8, out_dtype=alt.F32)
    h.gemm_adapters(d, x, w, ids, a, b, y, **ws(h.gemm_adapters_workspace_size(d)))
    g = alt.grouped_desc(M, 1, N, K, out_dtype=alt.F32)
    h.gemm_grouped(g, x, w, torch.tensor([0, M], dtype=torch.int32, device="cuda"), plain)
    none = ids < 0
    close(y[none], f64(plain[none]), 2 * K * EPS * (np.abs(f64(x[none])) @ np.abs(f64(w)).T))
    assert (y[~none] != plain[~none]).any()


@pytest.mark.parametrize("M,N", [(16, 128), (300, 640), (3000, 2048)])
def test_adapters_special_values_stay_with_their_rows(h, M, N):
    """An adapter full of NaN or infinities, and a row of x that holds one, reach their own rows only."""
    K, G, r = 256, 4, 16
    ids = torch.tensor(requests(M, G, 3, (1, 9)), dtype=torch.int32)
    x, w = matrix(normal(1, M, K), torch.bfloat16), matrix(normal(2, N, K, std=0.05), torch.bfloat16)
    a, b = matrix(normal(3, G * r, K), torch.bfloat16).view(G, r, K), matrix(normal(4, G * N, r), torch.bfloat16).view(G, N, r)
    d = alt.adapters_desc(M, N, K, G, r)
    space = ws(h.gemm_adapters_workspace_size(d))

    def run(x, a, b):
        y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
        h.gemm_adapters(d, x, w, ids.cuda(), a, b, y, **space)
        torch.cuda.synchronize()
        return y
    clean, bad_a, bad_b, bad_x = run(x, a, b), a.clone(), b.clone(), x.clone()
    bad_a[1, 3, 7], bad_b[2], bad_x[5, 9] = float("inf"), float("nan"), float("nan")
    got = run(bad_x, bad_a, bad_b)
    lost = (ids == 1) | (ids == 2)
    lost[5] = True
    assert torch.equal(got[~lost.cuda()], clean[~lost.cuda()])
    assert torch.isnan(got[(ids == 2).cuda()]).all() and torch.isnan(got[5]).all()


def test_adapters_without_rows(h):
    d = alt.adapters_desc(0, 32, 64, 2, 8)
    assert h.gemm_adapters_workspace_size(d) == 0
    h.gemm_adapters(d, None, None, None, None, None, None)


@pytest.mark.parametrize("M", [7, 500])
def test_adapters_captured_on_another_stream_and_replayed(h, M):
    N, K, G, r = 384, 512, 5, 16
    x, w = matrix(normal(1, M, K), torch.bfloat16), matrix(normal(2, N, K, std=0.05), torch.bfloat16)
    a, b = matrix(normal(3, G * r, K), torch.bfloat16).view(G, r, K), matrix(normal(4, G * N, r), torch.bfloat16).view(G, N, r)
    ids = torch.tensor(requests(M, G, 3, (1, 9)), dtype=torch.int32, device="cuda")
    d = alt.adapters_desc(M, N, K, G, r)
    y, space = torch.empty(M, N, dtype=torch.bfloat16, device="cuda"), ws(h.gemm_adapters_workspace_size(d))
    replayed(lambda: h.gemm_adapters(d, x, w, ids, a, b, y, **space), [y], lambda: y.fill_(3))
