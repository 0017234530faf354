"""Products of expert layers and of 8-bit layers, and the quantizer of rows, against plain sums in 64 bits.

Tolerances.  fp32 sums of n products, in any order: n * 2^-24 * sum |a||b| (the textbook bound), for the fused bias one rounding more;
sums of 8-bit products are exact and take three roundings (to fp32, and two scales), the bias a fourth: 4 * 2^-24 of the largest
intermediate value; a bf16 result one rounding more, 2^-8 of the value.  Quantized rows have one right answer."""
import numpy as np
import pytest
import torch

import paper_2210_12415_amd as alt

pytestmark = pytest.mark.gpu

TORCH = {alt.F32: torch.float32, alt.BF16: torch.bfloat16, alt.I8: torch.int8}
EPS = 2.0 ** -24


@pytest.fixture(scope="module")
def h():
    return alt.Handle()


class Canary:
    """A device matrix with unused columns and guard rows, all holding a pattern."""

    def __init__(self, rows, cols, dtype, stride=0, lead=()):
        self.rows, self.cols = rows, cols
        self.stride = stride or cols
        n = int(np.prod(lead, dtype=np.int64)) if lead else 1
        self.whole = torch.full((n * rows * self.stride + 256,), 77, dtype=dtype, device="cuda")
        self.at = self.whole[128:128 + n * rows * self.stride]
        self.t = self.at.view(*lead, rows, self.stride)[..., :cols]

    def data_ptr(self):
        return self.at.data_ptr()

    def untouched(self):
        edge = bool((self.whole[:128] == 77).all()) and bool((self.whole[-128:] == 77).all())
        pad = self.at.view(-1, self.stride)[:, self.cols:]
        return edge and bool((pad == 77).all())


def matrix(values, dtype, stride=0, offset=0):
    """A device matrix with `values` in rows `stride` apart (what lies between them is NaN, or 99 in 8 bits), `offset` elements into its buffer."""
    values = torch.as_tensor(values)
    rows, cols = values.shape[-2:]
    stride = stride or cols
    fill = 99 if dtype == torch.int8 else float("nan")
    buf = torch.full((int(np.prod(values.shape[:-1], dtype=np.int64)) * stride + offset,), fill, dtype=dtype, device="cuda")
    view = buf[offset:].view(*values.shape[:-1], stride)[..., :cols]
    view.copy_(values.to(dtype))
    return view


def f64(t):
    return t.cpu().double().numpy()


def normal(seed, *shape, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g) * std


def close(got, want, tol, what=""):
    got, want = f64(got), np.asarray(want)
    bad = ~(np.abs(got - want) <= tol)
    bad &= ~(np.isnan(got) & np.isnan(want))
    assert not bad.any(), "%s: %d of %d off, first at %s: %r for %r" % (what, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0])


# ---- quantizer -------------------------------------------------------------------------------------------------------------

def exact_rows(x):
    """The definition in 64 bits (x / s of a 24-bit by a 16-bit number is exact enough there to tell every tie)."""
    x = f64(x)
    top = np.abs(x).max(axis=1)
    with np.errstate(over="ignore"):
        m, e = np.frexp((top / 127.0).astype(np.float32).astype(np.float64))
    s = np.maximum(np.ldexp(np.ceil(m * 65536.0) / 65536.0, e), 2.0 ** -126)
    return np.rint(x / s[:, None]).astype(np.int8), s


def quantize(h, x, dtype, ldq=0):
    rows, cols = x.shape
    q, s = Canary(rows, cols, torch.int8, ldq), Canary(1, rows, torch.float32)
    h.quantize_rows(dtype, rows, cols, x, q, s, x_stride=x.stride(0) if rows > 1 else 0, q_stride=ldq)
    torch.cuda.synchronize()
    assert q.untouched() and s.untouched()
    return q.t, s.t[0]


@pytest.mark.parametrize("dtype", [alt.F32, alt.BF16])
@pytest.mark.parametrize("rows,cols,ldx,ldq", [(1, 1, 0, 0), (1, 7, 0, 0), (3, 8, 0, 0), (5, 63, 65, 71), (2, 768, 0, 0), (128, 768, 0, 0), (7, 2048, 0, 0),
                                               (9, 2049, 0, 0), (4, 4099, 4101, 4107), (1, 8192, 0, 0), (3, 8200, 8208, 0), (2, 20011, 0, 0), (3, 70000, 0, 0),
                                               (1000, 33, 0, 40)])
def test_quantize_rows(h, dtype, rows, cols, ldx, ldq):
    x = normal(rows * 7 + cols, rows, cols) * torch.exp(2 * normal(cols, rows, 1))
    x = matrix(x, TORCH[dtype], ldx, offset=1)
    q, s = quantize(h, x, dtype, ldq)
    want_q, want_s = exact_rows(x)
    assert np.array_equal(f64(s), want_s)
    assert np.array_equal(q.cpu().numpy(), want_q)


def test_quantize_rows_ties_extremes_and_specials(h):
    cols = 300
    half = torch.arange(cols) % 255 - 127.0
    rows = [torch.zeros(cols), torch.full((cols,), 3.0), half, half - 0.5 * (half > -127), (half + 0.5) * 2.0 ** -20, half * 2.0 ** -133, half * 2.0 ** -149,
            half * 2.0 ** 120, torch.cat([half[:-1], torch.tensor([127.5])])]
    rows.append(torch.full((cols,), 2.0 ** -149))
    rows.append(torch.full((cols,), torch.finfo(torch.float32).max))
    x = matrix(torch.stack(rows), torch.float32)
    q, s = quantize(h, x, alt.F32)
    want_q, want_s = exact_rows(x)
    assert np.array_equal(f64(s), want_s) and np.array_equal(q.cpu().numpy(), want_q)
    # rows with an infinity or a NaN: scale NaN, q zero, and their neighbours as ever
    bad = x.clone()
    for r, v in ((1, float("inf")), (3, float("-inf")), (5, float("nan"))):
        bad[r, (r * 97) % cols] = v
    q2, s2 = quantize(h, bad, alt.F32)
    lost = torch.tensor([r in (1, 3, 5) for r in range(len(rows))])
    assert torch.isnan(s2.cpu()[lost]).all() and (q2.cpu()[lost] == 0).all()
    assert torch.equal(q2.cpu()[~lost], q.cpu()[~lost]) and torch.equal(s2.cpu()[~lost], s.cpu()[~lost])


# ---- 8-bit product ---------------------------------------------------------------------------------------------------------

def scaled_reference(q, s, w, t, bias, relu):
    """(value, largest intermediate value) in 64 bits."""
    y = (f64(q) @ f64(w).T) * f64(s)[:, None] * f64(t)
    size = np.abs(y)
    if bias is not None:
        y = y + f64(bias)
        size = size + np.abs(f64(bias))
    return (np.maximum(y, 0) if relu else y), size


I8_SHAPES = [(1, 1, 1), (1, 64, 64), (1, 3072, 768), (2, 65, 16), (3, 17, 130), (16, 256, 1024), (17, 100, 333), (31, 129, 127), (33, 512, 48), (64, 64, 128),
             (65, 200, 2049), (100, 1000, 15), (128, 768, 3072), (200, 192, 256), (257, 513, 640), (513, 300, 1031)]


@pytest.mark.parametrize("M,N,K", I8_SHAPES)
@pytest.mark.parametrize("out,bias,relu,pad", [(alt.BF16, False, False, 0), (alt.F32, True, True, 0), (alt.F32, True, False, 16), (alt.BF16, True, True, 3)])
def test_gemm_i8(h, M, N, K, out, bias, relu, pad):
    g = torch.Generator().manual_seed(M * 31 + N * 7 + K)
    q = matrix(torch.randint(-128, 128, (M, K), generator=g), torch.int8, K + pad, offset=pad)
    w = matrix(torch.randint(-128, 128, (N, K), generator=g), torch.int8, K + pad, offset=pad)
    s, t = normal(1, M).abs().cuda() * 0.01, normal(2, N).abs().cuda() * 0.01
    b = normal(3, N).cuda() if bias else None
    y = Canary(M, N, TORCH[out], N + pad)
    d = alt.gemm_i8_desc(M, N, K, out_dtype=out, epilogue=(alt.EPI_BIAS if bias else 0) | (alt.EPI_RELU if relu else 0), lda=K + pad, ldb=K + pad, ldc=N + pad)
    need = h.gemm_i8_workspace_size(d)
    for ws in ([0, need] if need else [0]):
        y.t.fill_(55)
        h.gemm_i8(d, q, s, w, t, y, bias=b, workspace=torch.empty(ws, dtype=torch.uint8, device="cuda") if ws else None, ws_bytes=ws)
        torch.cuda.synchronize()
        assert y.untouched()
        want, size = scaled_reference(q, s, w, t, b, relu)
        close(y.t, want, 4 * EPS * size + (2.0 ** -8 * np.abs(want) if out == alt.BF16 else 0), "ws %d" % ws)


@pytest.mark.parametrize("M", [1, 16, 40, 200])
def test_gemm_i8_sums_are_exact(h, M):
    """Scales of powers of two and sums below 2^24: every output has one right value, also at the ends of the 8-bit range."""
    N, K = 96, 1000
    g = torch.Generator().manual_seed(M)
    q = torch.randint(-128, 128, (M, K), generator=g, dtype=torch.int32)
    w = torch.randint(-128, 128, (N, K), generator=g, dtype=torch.int32)
    q[0], w[0], w[1] = -128, -128, 127
    y = torch.empty(M, N, device="cuda")
    one = torch.full((M,), 0.5, device="cuda"), torch.full((N,), 4.0, device="cuda")
    h.gemm_i8(alt.gemm_i8_desc(M, N, K, out_dtype=alt.F32), matrix(q, torch.int8), one[0], matrix(w, torch.int8), one[1], y)
    assert torch.equal(y.cpu().double(), 2.0 * (q.double() @ w.double().T))


@pytest.mark.parametrize("M,N,pad", [(1, 64, 1), (16, 33, 0), (512, 1040, 1), (512, 1040, 17), (513, 1024, 0)])
def test_gemm_i8_longest_sums(h, M, N, pad):
    """The longest reduction of the largest products, of either sign (2147467264 and -2130690176; the fp32 of the exact sum is one value), in tiles of
    16 rows, whole chunks (131071 of 131072 bytes, laid out anew, among them) and any alignment."""
    K = 131071
    q, w = torch.full((M * (K + pad),), -128, dtype=torch.int8, device="cuda"), torch.full((N, K + pad), -128, dtype=torch.int8, device="cuda")
    w[1::2] = 127
    d = alt.gemm_i8_desc(M, N, K, out_dtype=alt.F32, lda=K + pad, ldb=K + pad)
    need = h.gemm_i8_workspace_size(d)
    want = torch.full((M, N), float(K * 128 * 128), device="cuda")
    want[:, 1::2] = float(-K * 128 * 127)
    for ws in ([0, need] if need else [0]):
        y = torch.zeros(M, N, device="cuda")
        h.gemm_i8(d, q, torch.ones(M, device="cuda"), w, torch.ones(N, device="cuda"), y, workspace=torch.empty(ws, dtype=torch.uint8, device="cuda") if ws else None,
                  ws_bytes=ws)
        assert torch.equal(y, want), ws


def test_gemm_i8_rows_without_a_scale_are_nan(h):
    q, w = torch.ones(20, 64, dtype=torch.int8, device="cuda"), torch.ones(32, 64, dtype=torch.int8, device="cuda")
    s, t = torch.ones(20, device="cuda"), torch.ones(32, device="cuda")
    s[3] = float("nan")
    y = torch.empty(20, 32, device="cuda")
    h.gemm_i8(alt.gemm_i8_desc(20, 32, 64, out_dtype=alt.F32, epilogue=alt.EPI_RELU), q, s, w, t, y)
    want = torch.full((20, 32), 64.0)
    want[3] = float("nan")
    assert torch.equal(torch.nan_to_num(y.cpu(), nan=-1.0), torch.nan_to_num(want, nan=-1.0))


# ---- products of groups ----------------------------------------------------------------------------------------------------

# (offsets, rows of the tensors): empty experts, rows of no expert before, behind and alone, single tokens, tiles that end inside
SPANS = [([0, 1], 1), ([0, 0, 0, 1, 1], 1), ([0, 3, 3, 20, 37, 37], 37), ([0, 64, 128, 192], 192), ([0, 65, 65, 66, 300], 300), ([5, 9, 100], 120), ([0, 0, 0], 13),
         ([13, 13], 13), ([0] + [i for i in range(1, 71)], 70), ([0] + [2 * i for i in range(1, 131)] + [300], 310), ([0, 500], 500), ([0, 16, 200, 217, 700], 700)]
SIZES = [(64, 64), (96, 200), (33, 17), (129, 1030), (515, 72), (256, 320), (1, 1), (8, 2049)]


def make_offsets(off):
    return torch.tensor(off, dtype=torch.int32, device="cuda")


def spans_of(off):
    return [(e, off[e], off[e + 1]) for e in range(len(off) - 1) if off[e + 1] > off[e]]


def cases():
    """Every span list with a size, every size with a span list, and all types and paddings among them."""
    out = []
    for i in range(24):
        off, rows = SPANS[i % len(SPANS)]
        n, k = SIZES[(i * 5 + i // 8) % len(SIZES)]
        out.append((off, rows, n, k, [alt.BF16, alt.F32][(i + i // 12) % 2], [0, 8, 3][i % 3]))
    return out


@pytest.mark.parametrize("off,rows,N,K,dtype,pad", cases())
def test_grouped_forward(h, off, rows, N, K, dtype, pad):
    E, td = len(off) - 1, TORCH[dtype]
    x = matrix(normal(1, rows, K), td, K + pad, offset=pad)
    w = matrix(normal(2, E, N, K, std=K ** -0.5), td, K + pad, offset=pad)
    bias = normal(3, E, N).cuda()
    offsets = make_offsets(off)
    for out, epi in ((alt.F32, 0), (alt.F32, alt.EPI_BIAS | alt.EPI_RELU)) + (((alt.BF16, alt.EPI_BIAS),) if dtype == alt.BF16 else ()):
        y = Canary(rows, N, TORCH[out], N + pad)
        d = alt.grouped_desc(rows, E, N, K, in_dtype=dtype, out_dtype=out, epilogue=epi, lda=K + pad, ldb=K + pad, ldc=N + pad)
        need = h.gemm_grouped_workspace_size(d)
        want, tol = np.zeros((rows, N)), np.zeros((rows, N))
        for e, lo, hi in spans_of(off):
            a, b = f64(x[lo:hi]), f64(w[e])
            want[lo:hi], tol[lo:hi] = a @ b.T, K * EPS * (np.abs(a) @ np.abs(b).T)
            if epi & alt.EPI_BIAS:
                want[lo:hi] += f64(bias[e])
                tol[lo:hi] += 2 * EPS * np.abs(want[lo:hi])
        if epi & alt.EPI_RELU:
            want = np.maximum(want, 0)
        if out == alt.BF16:
            tol += 2.0 ** -8 * np.abs(want)
        for ws in ([0, need] if need else [0]):
            y.t.fill_(55)
            h.gemm_grouped(d, x, w, offsets, y, bias=bias if epi & alt.EPI_BIAS else None,
                           workspace=torch.empty(ws, dtype=torch.uint8, device="cuda") if ws else None, ws_bytes=ws)
            torch.cuda.synchronize()
            assert y.untouched()
            close(y.t, want, tol, "out %d epilogue %d ws %d" % (out, epi, ws))


@pytest.mark.parametrize("off,rows,N,K", [(o, r) + SIZES[(i * 3) % len(SIZES)] for i, (o, r) in enumerate(SPANS)])
def test_grouped_forward_i8(h, off, rows, N, K):
    E, pad = len(off) - 1, [0, 16, 5][rows % 3]
    g = torch.Generator().manual_seed(rows)
    q = matrix(torch.randint(-127, 128, (rows, K), generator=g), torch.int8, K + pad)
    w = matrix(torch.randint(-127, 128, (E, N, K), generator=g), torch.int8, K + pad)
    s, t, bias = normal(1, rows).abs().cuda() * 0.01, normal(2, E, N).abs().cuda() * 0.01, normal(3, E, N).cuda()
    offsets = make_offsets(off)
    for out, relu in ((alt.F32, False), (alt.BF16, True)):
        y = Canary(rows, N, TORCH[out])
        d = alt.grouped_desc(rows, E, N, K, in_dtype=alt.I8, out_dtype=out, epilogue=alt.EPI_BIAS | (alt.EPI_RELU if relu else 0), lda=K + pad, ldb=K + pad)
        need = h.gemm_grouped_workspace_size(d)
        h.gemm_grouped(d, q, w, offsets, y, a_scale=s, b_scale=t, bias=bias, workspace=torch.empty(need, dtype=torch.uint8, device="cuda") if need else None, ws_bytes=need)
        torch.cuda.synchronize()
        assert y.untouched()
        want, tol = np.zeros((rows, N)), np.zeros((rows, N))
        for e, lo, hi in spans_of(off):
            want[lo:hi], size = scaled_reference(q[lo:hi], s[lo:hi], w[e], t[e], bias[e], relu)
            tol[lo:hi] = 4 * EPS * size + (2.0 ** -8 * np.abs(want[lo:hi]) if out == alt.BF16 else 0)
        close(y.t, want, tol, "out %d" % out)


@pytest.mark.parametrize("off,rows,N,K,dtype,pad", cases())
def test_grouped_gradients(h, off, rows, N, K, dtype, pad):
    E, td = len(off) - 1, TORCH[dtype]
    x = matrix(normal(1, rows, K).clamp_(min=0), td, K + pad, offset=pad)
    w = matrix(normal(2, E, N, K, std=K ** -0.5), td, K + pad, offset=pad)
    dy = matrix(normal(3, rows, N), td, N + pad, offset=pad)
    offsets = make_offsets(off)
    for out in (alt.F32, alt.BF16) if dtype == alt.BF16 else (alt.F32,):
        for mask in (False, True):
            dx = Canary(rows, K, TORCH[out], K + pad)
            d = alt.grouped_desc(rows, E, N, K, in_dtype=dtype, out_dtype=out, epilogue=alt.EPI_RELU if mask else 0, lda=K + pad, ldb=K + pad, ldc=N + pad)
            need = h.gemm_grouped_dx_workspace_size(d)
            h.gemm_grouped_dx(d, dy, w, offsets, dx, relu_of=x if mask else None, workspace=torch.empty(need, dtype=torch.uint8, device="cuda") if need else None,
                              ws_bytes=need)
            torch.cuda.synchronize()
            assert dx.untouched()
            want, tol = np.zeros((rows, K)), np.zeros((rows, K))
            for e, lo, hi in spans_of(off):
                g, b = f64(dy[lo:hi]), f64(w[e])
                want[lo:hi], tol[lo:hi] = g @ b, N * EPS * (np.abs(g) @ np.abs(b))
            if mask:
                want *= f64(x) > 0
            close(dx.t, want, tol + (2.0 ** -8 * np.abs(want) if out == alt.BF16 else 0), "dx out %d mask %d" % (out, mask))
        for with_bias in (True, False):
            dw, db = Canary(N, K, TORCH[out], K + pad, lead=(E,)), Canary(E, N, torch.float32)
            d = alt.grouped_desc(rows, E, N, K, in_dtype=dtype, out_dtype=out, epilogue=alt.EPI_BIAS if with_bias else 0, lda=K + pad, ldb=K + pad, ldc=N + pad)
            need = h.gemm_grouped_dw_workspace_size(d)
            want, tol = np.zeros((E, N, K)), np.zeros((E, N, K))
            want_b, tol_b = np.zeros((E, N)), np.zeros((E, N))
            for e, lo, hi in spans_of(off):
                g, a = f64(dy[lo:hi]), f64(x[lo:hi])
                want[e], tol[e] = g.T @ a, (hi - lo) * EPS * (np.abs(g).T @ np.abs(a))
                want_b[e], tol_b[e] = g.sum(axis=0), (hi - lo) * EPS * np.abs(g).sum(axis=0)
            for ws in ([0, need] if need else [0]):
                dw.t.fill_(55)
                db.t.fill_(77)
                h.gemm_grouped_dw(d, x, dy, offsets, dw, dbias=db if with_bias else None,
                                  workspace=torch.empty(ws, dtype=torch.uint8, device="cuda") if ws else None, ws_bytes=ws)
                torch.cuda.synchronize()
                assert dw.untouched() and db.untouched()
                close(dw.t, want, tol + (2.0 ** -8 * np.abs(want) if out == alt.BF16 else 0), "dw out %d ws %d" % (out, ws))
                if with_bias:
                    close(db.t, want_b, tol_b, "db")


def filled(shape, dtype, seed, offset=0):
    """A large operand of random values, `offset` elements into its buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = int(np.prod(shape))
    buf = torch.empty(n + offset, dtype=dtype, device="cuda")
    if dtype == torch.int8:
        buf.copy_(torch.randint(-127, 128, (n + offset,), generator=g, device="cuda"))
    else:
        buf.copy_(torch.randn(n + offset, generator=g, device="cuda"))
    return buf[offset:].view(shape)


def worst(got, want, size, n):
    """The largest error in units of n * 2^-24 of the sums of magnitudes."""
    return float(((got.double() - want).abs() / (n * EPS * size).clamp(min=1e-30)).max())


@pytest.mark.parametrize("M,N,K,offset", [(2049, 2051, 4099, 0), (2500, 2048, 4100, 3), (3000, 3001, 4096, 0)])
def test_large_8_bit_products_at_any_alignment(h, M, N, K, offset):
    """Without a workspace, with one in which the operands are laid out anew where that pays, and with one that starts anywhere: the same sums."""
    q, w = filled((M, K), torch.int8, 1, offset), filled((N, K), torch.int8, 2, offset)
    s, t = torch.ones(M, device="cuda"), torch.ones(N, device="cuda")
    want = q.double() @ w.double().T
    d = alt.gemm_i8_desc(M, N, K, out_dtype=alt.F32)
    need = h.gemm_i8_workspace_size(d)
    assert (need > 0) == (K % 16 != 0)
    ws = torch.empty(need + 64, dtype=torch.uint8, device="cuda")
    y = Canary(M, N, torch.float32)
    for at, nbytes in ((None, 0), (ws, need), (ws[5:], need), (ws, need // 2)):
        y.t.fill_(55)
        h.gemm_i8(d, q, s, w, t, y, workspace=at, ws_bytes=nbytes)
        torch.cuda.synchronize()
        assert y.untouched() and torch.equal(y.t.double(), want.float().double())


@pytest.mark.parametrize("off,N,K,offset", [([0, 700, 700, 2100, 3001], 1027, 2051, 0), ([0, 1500, 3000], 2047, 2050, 1), ([0, 2048, 4096], 2048, 2052, 0)])
def test_large_layers_at_any_alignment(h, off, N, K, offset):
    """Products and gradients with and without a workspace in which the operands are laid out anew."""
    rows, E = off[-1], len(off) - 1
    x, w, dy = filled((rows, K), torch.bfloat16, 1, offset), filled((E, N, K), torch.bfloat16, 2, offset), filled((rows, N), torch.bfloat16, 3, offset)
    o = make_offsets(off)
    d = alt.grouped_desc(rows, E, N, K, out_dtype=alt.F32)
    db = alt.grouped_desc(rows, E, N, K, out_dtype=alt.F32, epilogue=alt.EPI_BIAS)
    dm = alt.grouped_desc(rows, E, N, K, out_dtype=alt.F32, epilogue=alt.EPI_RELU)
    needs = h.gemm_grouped_workspace_size(d), h.gemm_grouped_dx_workspace_size(dm), h.gemm_grouped_dw_workspace_size(db)
    assert any(needs)
    ws = torch.empty(max(needs), dtype=torch.uint8, device="cuda")
    for use in (False, True):
        arg = [dict(workspace=ws, ws_bytes=n) if use and n else {} for n in needs]
        y, dx, dw, bias = Canary(rows, N, torch.float32), Canary(rows, K, torch.float32), Canary(N, K, torch.float32, lead=(E,)), torch.empty(E, N, device="cuda")
        h.gemm_grouped(d, x, w, o, y, **arg[0])
        h.gemm_grouped_dx(dm, dy, w, o, dx, relu_of=x, **arg[1])
        h.gemm_grouped_dw(db, x, dy, o, dw, dbias=bias, **arg[2])
        torch.cuda.synchronize()
        assert y.untouched() and dx.untouched() and dw.untouched()
        for e in range(E):
            lo, hi = off[e], off[e + 1]
            xd, wd, gd = x[lo:hi].double(), w[e].double(), dy[lo:hi].double()
            if hi == lo:
                assert not dw.t[e].any() and not bias[e].any()
                continue
            assert worst(y.t[lo:hi], xd @ wd.T, xd.abs() @ wd.abs().T, K) <= 1
            assert worst(dx.t[lo:hi], (gd @ wd) * (xd > 0), gd.abs() @ wd.abs(), N) <= 1
            assert worst(dw.t[e], gd.T @ xd, gd.abs().T @ xd.abs(), hi - lo) <= 1
            assert worst(bias[e], gd.sum(0), gd.abs().sum(0), hi - lo) <= 1


@pytest.mark.parametrize("off,N,K", [([0, 2304, 2305, 4700, 8192], 1024, 512), ([0, 300, 5000, 5100], 2304, 1024)])
@pytest.mark.parametrize("dtype", [alt.BF16, alt.I8])
def test_large_layers(h, off, N, K, dtype):
    """Tiles of both sizes, groups that end inside one."""
    rows, E, td = off[-1], len(off) - 1, TORCH[dtype]
    x, w = filled((rows, K), td, 1), filled((E, N, K), td, 2)
    o, y = make_offsets(off), Canary(rows, N, torch.float32)
    one = dict(a_scale=torch.ones(rows, device="cuda"), b_scale=torch.ones(E, N, device="cuda")) if dtype == alt.I8 else {}
    h.gemm_grouped(alt.grouped_desc(rows, E, N, K, in_dtype=dtype, out_dtype=alt.F32), x, w, o, y, **one)
    torch.cuda.synchronize()
    assert y.untouched()
    for e in range(E):
        lo, hi = off[e], off[e + 1]
        xd, wd = x[lo:hi].double(), w[e].double()
        assert worst(y.t[lo:hi], xd @ wd.T, xd.abs() @ wd.abs().T, K) <= 1
    if dtype == alt.I8:
        return
    dy = filled((rows, N), td, 3)
    d = alt.grouped_desc(rows, E, N, K, out_dtype=alt.F32, epilogue=alt.EPI_BIAS)
    dx, dw, bias = Canary(rows, K, torch.float32), Canary(N, K, torch.float32, lead=(E,)), torch.empty(E, N, device="cuda")
    h.gemm_grouped_dx(alt.grouped_desc(rows, E, N, K, out_dtype=alt.F32), dy, w, o, dx)
    h.gemm_grouped_dw(d, x, dy, o, dw, dbias=bias)
    torch.cuda.synchronize()
    assert dx.untouched() and dw.untouched()
    for e in range(E):
        lo, hi = off[e], off[e + 1]
        xd, wd, gd = x[lo:hi].double(), w[e].double(), dy[lo:hi].double()
        assert worst(dx.t[lo:hi], gd @ wd, gd.abs() @ wd.abs(), N) <= 1
        assert worst(dw.t[e], gd.T @ xd, gd.abs().T @ xd.abs(), hi - lo) <= 1
        assert worst(bias[e], gd.sum(0), gd.abs().sum(0), hi - lo) <= 1


@pytest.mark.parametrize("rows", [24, 500])
def test_gradients_against_differences(h, rows):
    """L = sum y * g is linear in x, w and bias, so a difference over any step is the derivative: along a random direction of each operand the
    differences of forward products equal the products with the gradients, but for the roundings of their fp32 sums (n * 2^-24 each)."""
    off, E, N, K = [0, 7, 7, rows], 3, 70, 90
    x, w, b, g = normal(1, rows, K).cuda(), normal(2, E, N, K).cuda(), normal(3, E, N).cuda(), normal(4, rows, N).cuda()
    ox, ow, ob = normal(5, rows, K).cuda(), normal(6, E, N, K).cuda(), normal(7, E, N).cuda()
    offsets = make_offsets(off)
    d = alt.grouped_desc(rows, E, N, K, in_dtype=alt.F32, out_dtype=alt.F32, epilogue=alt.EPI_BIAS)
    plain = alt.grouped_desc(rows, E, N, K, in_dtype=alt.F32, out_dtype=alt.F32)

    def loss(x, w, b):
        y = torch.empty(rows, N, device="cuda")
        h.gemm_grouped(d, x, w, offsets, y, bias=b)
        return float((y.double() * g.double()).sum()), float((y.double() * g.double()).abs().sum())
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    h.gemm_grouped_dx(plain, g, w, offsets, dx)
    h.gemm_grouped_dw(d, x, g, offsets, dw, dbias=db)
    for got, (up, down) in (((dx.double() * ox.double()).sum(), ((x + ox, w, b), (x - ox, w, b))), ((dw.double() * ow.double()).sum(), ((x, w + ow, b), (x, w - ow, b))),
                            ((db.double() * ob.double()).sum(), ((x, w, b + ob), (x, w, b - ob)))):
        (hi, size_hi), (lo, size_lo) = loss(*up), loss(*down)
        # each y is off by K * 2^-24 of sums that are K^0.5 times larger than itself at most here, and so is the gradient by its own
        assert abs(float(got) - (hi - lo) / 2) <= (rows + K + N) * EPS * 10 * (size_hi + size_lo)


@pytest.mark.parametrize("dtype", [alt.F32, alt.BF16, alt.I8])
def test_values_of_one_expert_stay_there(h, dtype):
    """Infinities and NaN in an expert's rows or weights reach that expert's results alone."""
    off, E, N, K = [0, 5, 40, 45, 80], 4, 72, 96
    rows, offsets = off[-1], make_offsets([0, 5, 40, 45, 80])
    if dtype == alt.I8:
        s = torch.ones(rows, device="cuda")
        s[5:40] = float("nan")
        t = torch.ones(E, N, device="cuda")
        t[3] = float("inf")
        x, w = torch.ones(rows, K, dtype=torch.int8, device="cuda"), torch.ones(E, N, K, dtype=torch.int8, device="cuda")
        y = torch.empty(rows, N, device="cuda")
        h.gemm_grouped(alt.grouped_desc(rows, E, N, K, in_dtype=dtype, out_dtype=alt.F32), x, w, offsets, y, a_scale=s, b_scale=t)
        y = y.cpu()
        assert torch.isnan(y[5:40]).all() and torch.isinf(y[45:]).all() and (y[:5] == K).all() and (y[40:45] == K).all()
        return
    x, w = normal(1, rows, K), normal(2, E, N, K)
    x[5:40, 3] = float("nan")
    w[3] = float("inf")
    x, w = matrix(x, TORCH[dtype]), matrix(w, TORCH[dtype])
    dy = matrix(normal(3, rows, N), TORCH[dtype])
    y, dx, dw = torch.empty(rows, N, device="cuda"), torch.empty(rows, K, device="cuda"), torch.empty(E, N, K, device="cuda")
    d = alt.grouped_desc(rows, E, N, K, in_dtype=dtype, out_dtype=alt.F32)
    h.gemm_grouped(d, x, w, offsets, y)
    h.gemm_grouped_dx(d, dy, w, offsets, dx)
    h.gemm_grouped_dw(d, x, dy, offsets, dw)
    y, dx, dw = y.cpu(), dx.cpu(), dw.cpu()
    ok = torch.isfinite
    assert torch.isnan(y[5:40]).all() and not ok(y[45:]).any() and ok(y[:5]).all() and ok(y[40:45]).all()
    assert ok(dx[:45]).all() and not ok(dx[45:]).any()
    assert torch.isnan(dw[1, :, 3]).all() and ok(dw[[0, 2, 3]]).all() and ok(dw[1, :, [0, 95]]).all()


@pytest.mark.parametrize("off", [[-5, 20, 10 ** 9], [40, 10, 30], [2 ** 31 - 1, -2 ** 31, 7]])
def test_offsets_out_of_range_stay_in_the_buffers(h, off):
    rows, E, N, K = 40, 2, 70, 64
    x, w, dy = normal(1, rows, K).bfloat16().cuda(), normal(2, E, N, K).bfloat16().cuda(), normal(3, rows, N).bfloat16().cuda()
    y, dx, dw = Canary(rows, N, torch.float32), Canary(rows, K, torch.float32), Canary(N, K, torch.float32, lead=(E,))
    d, o = alt.grouped_desc(rows, E, N, K, out_dtype=alt.F32), make_offsets(off)
    h.gemm_grouped(d, x, w, o, y)
    h.gemm_grouped_dx(d, dy, w, o, dx)
    h.gemm_grouped_dw(d, x, dy, o, dw)
    torch.cuda.synchronize()
    assert y.untouched() and dx.untouched() and dw.untouched()
    assert torch.isfinite(dw.t).all()


DISORDER = {"alternating": lambda rows, E: [(i % 2) * rows for i in range(E + 1)], "falling": lambda rows, E: [rows - i * rows // E for i in range(E + 1)],
            "anywhere": lambda rows, E: np.random.default_rng(rows).integers(-2 ** 31, 2 ** 31, E + 1).tolist(),
            "shuffled": lambda rows, E: np.random.default_rng(E).integers(0, rows + 1, E + 1).tolist()}


@pytest.mark.parametrize("disorder", sorted(DISORDER))
@pytest.mark.parametrize("rows,E,N,K", [(900, 70, 64, 128), (2500, 100, 136, 128), (2500, 100, 130, 130), (35840, 70, 4096, 128)],
                         ids=["tiles_of_16", "whole_chunks", "any_alignment", "large_tiles"])
def test_offsets_out_of_order_count_as_their_running_maximum(h, rows, E, N, K, disorder):
    """Whatever the offsets hold, every row is one expert's or none's, and is computed once; all sums exact.  (The gradient by the weights takes an
    expert's own two offsets.)"""
    off = DISORDER[disorder](rows, E)
    x, w, dy = small_integers((rows, K), torch.bfloat16, 1), small_integers((E, N, K), torch.bfloat16, 2), small_integers((rows, N), torch.bfloat16, 3)
    y, dx, dw = Canary(rows, N, torch.float32), Canary(rows, K, torch.float32), Canary(N, K, torch.float32, lead=(E,))
    d, o = alt.grouped_desc(rows, E, N, K, out_dtype=alt.F32), make_offsets(off)
    h.gemm_grouped(d, x, w, o, y)
    h.gemm_grouped_dx(d, dy, w, o, dx)
    if rows < 10000:
        h.gemm_grouped_dw(d, x, dy, o, dw)
    torch.cuda.synchronize()
    assert y.untouched() and dx.untouched() and dw.untouched()
    at = np.maximum.accumulate(np.clip(off, 0, rows)).tolist()
    assert not y.t[:at[0]].any() and not y.t[at[E]:].any() and not dx.t[:at[0]].any() and not dx.t[at[E]:].any()
    for e, lo, hi in spans_of(at):
        assert torch.equal(y.t[lo:hi], x[lo:hi].float() @ w[e].float().T) and torch.equal(dx.t[lo:hi], dy[lo:hi].float() @ w[e].float()), e
    for e in range(E if rows < 10000 else 0):
        lo, hi = min(max(off[e], 0), rows), min(max(off[e + 1], 0), rows)
        assert torch.equal(dw.t[e], dy[lo:hi].float().T @ x[lo:hi].float()), e


@pytest.mark.parametrize("disorder", sorted(DISORDER))
@pytest.mark.parametrize("rows,E,N,K", [(60, 3000, 64, 128), (3500, 230, 64, 128), (9000, 230, 136, 128), (9000, 230, 130, 130)],
                         ids=["a_slot_for_a_row", "tiles_of_16", "whole_chunks", "any_alignment"])
def test_offsets_out_of_order_of_many_experts(h, rows, E, N, K, disorder):
    """Where a search finds the tiles: nothing outside the buffers, and of each row nothing but some expert's values, or zeros, or what was there."""
    off = DISORDER[disorder](rows, E)
    x, w, dy = small_integers((rows, K), torch.bfloat16, 1), small_integers((E, N, K), torch.bfloat16, 2), small_integers((rows, N), torch.bfloat16, 3)
    y, dx, dw = Canary(rows, N, torch.float32), Canary(rows, K, torch.float32), Canary(N, K, torch.float32, lead=(E,))
    d, o = alt.grouped_desc(rows, E, N, K, out_dtype=alt.F32), make_offsets(off)
    h.gemm_grouped(d, x, w, o, y)
    h.gemm_grouped_dx(d, dy, w, o, dx)
    h.gemm_grouped_dw(d, x, dy, o, dw)
    torch.cuda.synchronize()
    assert y.untouched() and dx.untouched() and dw.untouched()
    for got, most in ((y.t, 9 * K), (dx.t, 9 * N)):
        assert bool((got.abs() <= most).all()) and torch.equal(got, got.round())


@pytest.mark.parametrize("most,E,N,K,dtype", [(1, 63, 64, 64, alt.BF16), (3, 63, 70, 66, alt.F32), (1, 1000, 40, 72, alt.BF16), (1, 5000, 24, 32, alt.I8), (40, 100, 100, 64, alt.BF16), (40, 190, 48, 64, alt.BF16), (40, 191, 48, 66, alt.BF16), (300, 191, 64, 128, alt.BF16),
                                              (40, 1000, 33, 17, alt.I8), (40, 1000, 64, 72, alt.BF16), (90, 300, 33, 70, alt.BF16), (90, 300, 20, 36, alt.F32), (300, 200, 64, 64, alt.I8),
                                              (1, 1 << 20, 8, 8, alt.BF16), (2, 1 << 20, 8, 8, alt.I8)])
def test_many_experts(h, most, E, N, K, dtype):
    """More experts than a wave scans at once, of 0 to `most` rows, with rows of no expert before and behind; all sums exact."""
    counts = np.random.default_rng(E + most).integers(0, most + 1, E)
    counts[[0, E // 3, E // 2, E - 1]] = [most, 0, 0, 0]
    off = np.concatenate([[0], np.cumsum(counts)]) + 5
    rows, td = int(off[-1]) + 7, TORCH[dtype]
    expert = torch.as_tensor(np.concatenate([np.full(5, -1), np.repeat(np.arange(E), counts), np.full(7, -1)]), device="cuda")
    x, w, dy = small_integers((rows, K), td, 1), small_integers((E, N, K), td, 2), small_integers((rows, N), td, 3)
    y, o = Canary(rows, N, torch.float32), torch.as_tensor(off.astype(np.int32), device="cuda")
    one = dict(a_scale=torch.ones(rows, device="cuda"), b_scale=torch.ones(E, N, device="cuda")) if dtype == alt.I8 else {}
    d = alt.grouped_desc(rows, E, N, K, in_dtype=dtype, out_dtype=alt.F32)
    h.gemm_grouped(d, x, w, o, y, **one)
    dx = Canary(rows, K, torch.float32)
    if dtype != alt.I8:
        h.gemm_grouped_dx(d, dy, w, o, dx)
    torch.cuda.synchronize()
    assert y.untouched() and dx.untouched()
    for lo in range(0, rows, 20000):
        part = slice(lo, lo + 20000)
        own = w[expert[part].clamp(min=0)].float() * (expert[part] >= 0)[:, None, None]
        assert torch.equal(y.t[part], (own * x[part, None, :].float()).sum(2))
        if dtype != alt.I8:
            assert torch.equal(dx.t[part], (own * dy[part, :, None].float()).sum(1))


@pytest.mark.parametrize("E,mean,N,K,dtype", [(70, 500, 2048, 512, alt.BF16), (130, 500, 1024, 1024, alt.I8), (130, 500, 1024, 1024, alt.BF16), (2100, 240, 1024, 64, alt.BF16)])
def test_large_tiles_of_many_experts(h, E, mean, N, K, dtype):
    """Groups that end anywhere in a tile, empty ones, rows of no expert before and behind, in large tiles and the small ones at their ends; all sums exact."""
    counts = np.random.default_rng(E).integers(0, 2 * mean, E)
    counts[[0, 1, 2, 3, 4, 5, 62, 63, 64, E - 1]] = [256, 0, 1, 128, 129, 511, 0, 255, 0, 384]
    counts = counts * (E * mean) // counts.sum()
    off = np.concatenate([[0], np.cumsum(counts)]) + 130
    off, rows, td = off.tolist(), int(off[-1]) + 300, TORCH[dtype]
    x, w, y = small_integers((rows, K), td, 1), small_integers((E, N, K), td, 2), Canary(rows, N, torch.float32)
    one = dict(a_scale=torch.ones(rows, device="cuda"), b_scale=torch.ones(E, N, device="cuda")) if dtype == alt.I8 else {}
    d, o = alt.grouped_desc(rows, E, N, K, in_dtype=dtype, out_dtype=alt.F32), make_offsets(off)
    h.gemm_grouped(d, x, w, o, y, **one)
    torch.cuda.synchronize()
    assert y.untouched() and not y.t[:130].any() and not y.t[off[-1]:].any()
    for e, lo, hi in spans_of(off):
        assert torch.equal(y.t[lo:hi], x[lo:hi].float() @ w[e].float().T), e
    if dtype == alt.I8:
        return
    dy, dx = small_integers((rows, N), td, 3), Canary(rows, K, torch.float32)
    del y
    h.gemm_grouped_dx(d, dy, w, o, dx)
    torch.cuda.synchronize()
    assert dx.untouched() and not dx.t[:130].any() and not dx.t[off[-1]:].any()
    for e, lo, hi in spans_of(off):
        assert torch.equal(dx.t[lo:hi], dy[lo:hi].float() @ w[e].float()), e


def test_no_rows(h):
    E, N, K = 3, 64, 64
    o = make_offsets([0, 0, 0, 0])
    d = alt.grouped_desc(0, E, N, K, out_dtype=alt.F32, epilogue=alt.EPI_BIAS)
    h.gemm_grouped(d, None, None, o, None)
    dw, db = torch.ones(E, N, K, device="cuda"), torch.ones(E, N, device="cuda")
    h.gemm_grouped_dw(d, None, None, o, dw, dbias=db)
    assert not dw.any() and not db.any()
    h.quantize_rows(alt.F32, 0, 8, None, None, None)
    h.gemm_i8(alt.gemm_i8_desc(0, 8, 8), None, None, None, None, None)


def test_streams_and_graphs(h):
    """A layer on a stream of its own, and captured: every replay equals the eager pass, with other inputs and offsets each time."""
    rows, E, N, K = 48, 4, 192, 128
    x, w = normal(1, rows, K).bfloat16().cuda(), normal(2, E, N, K).bfloat16().cuda()
    o = make_offsets([0, 10, 11, 40, 48])
    y, dx, dw = torch.empty(rows, N, device="cuda"), torch.empty(rows, K, device="cuda"), torch.empty(E, N, K, device="cuda")
    q, s, wq = torch.empty(rows, K, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(E, N, K, dtype=torch.int8, device="cuda")
    t = torch.empty(E, N, device="cuda")
    y8 = torch.empty(rows, N, device="cuda")
    h.quantize_rows(alt.BF16, E * N, K, w, wq, t)
    d = alt.grouped_desc(rows, E, N, K, out_dtype=alt.F32)
    d8 = alt.grouped_desc(rows, E, N, K, in_dtype=alt.I8, out_dtype=alt.F32)
    dy = normal(3, rows, N).bfloat16().cuda()
    ws = {}
    for name, size in (("y", h.gemm_grouped_workspace_size(d)), ("dx", h.gemm_grouped_dx_workspace_size(d)), ("dw", h.gemm_grouped_dw_workspace_size(d))):
        ws[name] = dict(workspace=torch.empty(size, dtype=torch.uint8, device="cuda") if size else None, ws_bytes=size)

    def step():
        h.gemm_grouped(d, x, w, o, y, **ws["y"])
        h.gemm_grouped_dx(d, dy, w, o, dx, **ws["dx"])
        h.gemm_grouped_dw(d, x, dy, o, dw, **ws["dw"])
        h.quantize_rows(alt.BF16, rows, K, x, q, s)
        h.gemm_grouped(d8, q, wq, o, y8, a_scale=s, b_scale=t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i, off in enumerate(([0, 10, 11, 40, 48], [0, 0, 0, 0, 0], [0, 48, 48, 48, 48], [3, 4, 5, 6, 7])):
        x.copy_(normal(10 + i, rows, K))
        o.copy_(make_offsets(off))
        step()
        eager = [v.clone() for v in (y, dx, dw, y8)]
        for v in (y, dx, dw, y8):
            v.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, (y, dx, dw, y8)):
            assert torch.equal(a, b), i


def test_results_repeat(h):
    """The same call gives the same bits."""
    off, E, N, K = [0, 300, 301, 2000], 3, 200, 264
    x, w, dy = normal(1, 2000, K).bfloat16().cuda(), normal(2, E, N, K).bfloat16().cuda(), normal(3, 2000, N).bfloat16().cuda()
    o, d = make_offsets(off), alt.grouped_desc(2000, E, N, K, out_dtype=alt.F32, epilogue=alt.EPI_BIAS)
    need = h.gemm_grouped_dw_workspace_size(d)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    first = None
    for _ in range(4):
        dw, db = torch.empty(E, N, K, device="cuda"), torch.empty(E, N, device="cuda")
        h.gemm_grouped_dw(d, x, dy, o, dw, dbias=db, workspace=ws, ws_bytes=need)
        torch.cuda.synchronize()
        first = first or (dw, db)
        assert torch.equal(dw, first[0]) and torch.equal(db, first[1])


def small_integers(shape, dtype, seed):
    """Values of -3 .. 3: sums of a few thousand products of them are exact in 32 bits, in any order."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-3, 4, shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("red", [8, 64, 72, 136, 192, 264, 320, 400])
@pytest.mark.parametrize("dtype", [alt.BF16, alt.I8])
def test_large_tiles_with_any_number_of_steps(h, dtype, red):
    """Fewer steps of the reduction than the loads run ahead, as many, and some more; all sums exact."""
    M, N, td = 4093, 4096, TORCH[dtype]
    red *= 2 if dtype == alt.I8 else 1
    o = make_offsets([0, M])
    x, w, y = small_integers((M, red), td, 1), small_integers((1, N, red), td, 2), Canary(M, N, torch.float32)
    one = dict(a_scale=torch.ones(M, device="cuda"), b_scale=torch.ones(N, device="cuda")) if dtype == alt.I8 else {}
    h.gemm_grouped(alt.grouped_desc(M, 1, N, red, in_dtype=dtype, out_dtype=alt.F32), x, w, o, y, **one)
    torch.cuda.synchronize()
    assert y.untouched() and torch.equal(y.t, x.float() @ w[0].float().T)
    if dtype == alt.I8:
        return
    dy, w, dx = small_integers((M, red), td, 3), small_integers((1, red, N), td, 4), Canary(M, N, torch.float32)
    h.gemm_grouped_dx(alt.grouped_desc(M, 1, red, N, out_dtype=alt.F32), dy, w, o, dx)
    torch.cuda.synchronize()
    assert dx.untouched() and torch.equal(dx.t, dy.float() @ w[0].float())
    x, dy, dw, db = small_integers((red, 4088), td, 5), small_integers((red, N), td, 6), Canary(N, 4088, torch.float32), torch.empty(N, device="cuda")
    h.gemm_grouped_dw(alt.grouped_desc(red, 1, N, 4088, out_dtype=alt.F32, epilogue=alt.EPI_BIAS), x, dy, make_offsets([0, red]), dw, dbias=db)
    torch.cuda.synchronize()
    assert dw.untouched() and torch.equal(dw.t, dy.float().T @ x.float()) and torch.equal(db, dy.float().sum(0))


def far_apart(rows, cols, stride, dtype, seed, offset=0):
    """Rows `stride` elements apart in a buffer of more than 4 GiB, of which only they are written."""
    buf = torch.empty(rows * stride + offset, dtype=dtype, device="cuda")
    assert buf.numel() * buf.element_size() > 1 << 32
    view = buf[offset:].view(rows, stride)[:, :cols]
    view.copy_(small_integers((rows, cols), dtype, seed))
    return view


@pytest.mark.parametrize("rows,stride,offset", [(1030, 1 << 22, 0), (1030, (1 << 22) - 5, 3), (17, 1 << 22, 0)])
def test_operands_beyond_32_bits(h, rows, stride, offset):
    """Rows of every operand in buffers of more than 4 GiB (the few rows' weights are what is far apart there)."""
    N, K = (40, 72) if rows > 32 else (1030, 72)
    x8 = far_apart(rows, K, stride, torch.int8, 1, offset) if rows > 32 else small_integers((rows, K), torch.int8, 1)
    w8 = far_apart(N, K, stride, torch.int8, 2, offset) if N > 1024 else small_integers((N, K), torch.int8, 2)
    y = torch.empty(rows, N, device="cuda")
    d = alt.gemm_i8_desc(rows, N, K, out_dtype=alt.F32, lda=x8.stride(0), ldb=w8.stride(0))
    h.gemm_i8(d, x8, torch.ones(rows, device="cuda"), w8, torch.ones(N, device="cuda"), y)
    torch.cuda.synchronize()
    assert torch.equal(y, x8.float() @ w8.float().T)
    del x8, w8
    if rows <= 32:
        return
    rows, x, w = 600, small_integers((600, K), torch.bfloat16, 3), small_integers((2, N, K), torch.bfloat16, 4)
    o, far = make_offsets([0, 250, 600]), far_apart(600, N, stride, torch.bfloat16, 5, offset)
    want = torch.cat([x[:250].float() @ w[0].float().T, x[250:].float() @ w[1].float().T])
    h.gemm_grouped(alt.grouped_desc(rows, 2, N, K, ldc=stride), x, w, o, far)
    torch.cuda.synchronize()
    assert torch.equal(far.float(), want.bfloat16().float())
    far.copy_(small_integers((rows, N), torch.bfloat16, 6))
    dx, dw = torch.empty(rows, K, device="cuda"), torch.empty(2, N, K, device="cuda")
    d = alt.grouped_desc(rows, 2, N, K, out_dtype=alt.F32, ldc=stride)
    h.gemm_grouped_dx(d, far, w, o, dx)
    h.gemm_grouped_dw(d, x, far, o, dw)
    torch.cuda.synchronize()
    for e, (lo, hi) in enumerate(((0, 250), (250, 600))):
        assert torch.equal(dx[lo:hi], far[lo:hi].float() @ w[e].float()) and torch.equal(dw[e], far[lo:hi].float().T @ x[lo:hi].float())


def test_weights_beyond_32_bits(h):
    """An expert whose weights begin behind 4 GiB, with all three products of its layer."""
    E, N, K, rows = 34, 8192, 8192, 300
    w = torch.empty(E, N, K, dtype=torch.bfloat16, device="cuda")
    assert w.numel() * 2 > 1 << 32
    off = [0] * (E - 1) + [100, 300]
    for e in (E - 2, E - 1):
        w[e] = small_integers((N, K), torch.bfloat16, e)
    x, dy, o = small_integers((rows, K), torch.bfloat16, 1), small_integers((rows, N), torch.bfloat16, 2), make_offsets(off)
    y, dx = torch.empty(rows, N, device="cuda"), torch.empty(rows, K, device="cuda")
    d = alt.grouped_desc(rows, E, N, K, out_dtype=alt.F32)
    h.gemm_grouped(d, x, w, o, y)
    h.gemm_grouped_dx(d, dy, w, o, dx)
    torch.cuda.synchronize()
    for e, lo, hi in ((E - 2, 0, 100), (E - 1, 100, 300)):
        assert torch.equal(y[lo:hi], x[lo:hi].float() @ w[e].float().T) and torch.equal(dx[lo:hi], dy[lo:hi].float() @ w[e].float())
    del w
    dw = torch.full((E, N, K), 3, dtype=torch.bfloat16, device="cuda")
    h.gemm_grouped_dw(alt.grouped_desc(rows, E, N, K), x, dy, o, dw)
    torch.cuda.synchronize()
    assert not dw[:E - 2].any()
    for e, lo, hi in ((E - 2, 0, 100), (E - 1, 100, 300)):
        assert torch.equal(dw[e].float(), (dy[lo:hi].float().T @ x[lo:hi].float()).bfloat16().float())


def test_quantize_rows_beyond_32_bits(h):
    rows, cols, stride = 1030, 70, 1 << 22
    x = far_apart(rows, cols, stride, torch.bfloat16, 7)
    x[:, 1] = 3
    q = torch.empty(rows * stride, dtype=torch.int8, device="cuda").view(rows, stride)[:, :cols]
    s = torch.empty(rows, device="cuda")
    h.quantize_rows(alt.BF16, rows, cols, x, q, s, x_stride=stride, q_stride=stride)
    torch.cuda.synchronize()
    want, scale = exact_rows(x)
    assert np.array_equal(q.cpu().numpy(), want) and np.array_equal(f64(s), scale)


TILES = [([300], 1030, 272), ([1100], 1100, 256), ([1500], 1501, 528), ([40] * 40, 520, 256), ([33, 0, 700, 1, 129, 640], 1000, 144)]


@pytest.mark.parametrize("counts,N,K", TILES, ids=["one_group", "one_round", "two_rounds", "many_groups", "uneven"])
@pytest.mark.parametrize("pad", [0, 16, 1])
@pytest.mark.parametrize("dtype", [alt.BF16, alt.F32, alt.I8])
def test_tiles_of_every_size(h, counts, N, K, pad, dtype):
    """More rows than tiles of 16 are for, at strides of whole chunks and not, with bias and ReLU; all sums exact."""
    td, E, rows = TORCH[dtype], len(counts), sum(counts)
    off = [0]
    for c in counts:
        off.append(off[-1] + c)
    o, bias = make_offsets(off), torch.randint(-50, 50, (E, N), device="cuda").float()
    x, w = matrix(small_integers((rows, K), torch.float32, 1), td, K + pad), matrix(small_integers((E, N, K), torch.float32, 2), td, K + pad)
    one = dict(a_scale=torch.ones(rows, device="cuda"), b_scale=torch.ones(E, N, device="cuda")) if dtype == alt.I8 else {}
    y = Canary(rows, N, torch.float32, N + pad)
    d = alt.grouped_desc(rows, E, N, K, in_dtype=dtype, out_dtype=alt.F32, epilogue=alt.EPI_BIAS | alt.EPI_RELU, lda=K + pad, ldb=K + pad, ldc=N + pad)
    h.gemm_grouped(d, x, w, o, y, bias=bias, **one)
    torch.cuda.synchronize()
    assert y.untouched()
    for e in range(E):
        lo, hi = off[e], off[e + 1]
        assert torch.equal(y.t[lo:hi], torch.relu(x[lo:hi].float() @ w[e].float().T + bias[e])), e
    if dtype == alt.I8:
        return
    dy = matrix(small_integers((rows, N), torch.float32, 3), td, N + pad)
    dx, dw, db = Canary(rows, K, torch.float32, K + pad), Canary(N, K, torch.float32, K + pad, lead=(E,)), torch.empty(E, N, device="cuda")
    shape = dict(in_dtype=dtype, out_dtype=alt.F32, lda=K + pad, ldb=K + pad, ldc=N + pad)
    h.gemm_grouped_dx(alt.grouped_desc(rows, E, N, K, epilogue=alt.EPI_RELU, **shape), dy, w, o, dx, relu_of=x)
    h.gemm_grouped_dw(alt.grouped_desc(rows, E, N, K, epilogue=alt.EPI_BIAS, **shape), x, dy, o, dw, dbias=db)
    torch.cuda.synchronize()
    assert dx.untouched() and dw.untouched()
    for e in range(E):
        lo, hi = off[e], off[e + 1]
        assert torch.equal(dx.t[lo:hi], (dy[lo:hi].float() @ w[e].float()) * (x[lo:hi] > 0)), e
        assert torch.equal(dw.t[e], dy[lo:hi].float().T @ x[lo:hi].float()) and torch.equal(db[e], dy[lo:hi].float().sum(0)), e


@pytest.mark.parametrize("dtype", [alt.F32, alt.BF16])
@pytest.mark.parametrize("cols,ldx", [(1000, 0), (1025, 0), (1999, 2003), (2048, 0), (2056, 0)])
def test_quantize_many_rows(h, dtype, cols, ldx):
    x = matrix(normal(cols, 515, cols) * torch.exp(normal(7, 515, 1)), TORCH[dtype], ldx)
    q, s = quantize(h, x, dtype)
    want, scale = exact_rows(x)
    assert np.array_equal(q.cpu().numpy(), want) and np.array_equal(f64(s), scale)


@pytest.mark.parametrize("counts,N,K", [([1], 3742, 170), ([19], 2538, 64), ([2, 0, 33, 1], 77, 65), ([5] * 70, 130, 63), ([16, 17], 1000, 3), ([40], 31, 127)])
@pytest.mark.parametrize("pad", [0, 1, 8])
@pytest.mark.parametrize("dtype", [alt.BF16, alt.F32])
def test_gradient_by_few_rows(h, counts, N, K, pad, dtype):
    """Fewer columns than a tile's, tiles moved back to end with the matrix, reductions that end inside a unit; rows of no expert; all sums exact."""
    td, E, rows = TORCH[dtype], len(counts), sum(counts) + 3
    off = [2]
    for c in counts:
        off.append(off[-1] + c)
    x = matrix(small_integers((rows, K), torch.float32, 1), td, K + pad)
    w = matrix(small_integers((E, N, K), torch.float32, 2), td, K + pad)
    dy = matrix(small_integers((rows, N), torch.float32, 3), td, N + pad)
    for epilogue, out in ((alt.EPI_RELU, alt.F32), (0, alt.F32), (alt.EPI_RELU, dtype)):
        dx = Canary(rows, K, TORCH[out], K + pad)
        d = alt.grouped_desc(rows, E, N, K, in_dtype=dtype, out_dtype=out, epilogue=epilogue, lda=K + pad, ldb=K + pad, ldc=N + pad)
        h.gemm_grouped_dx(d, dy, w, make_offsets(off), dx, relu_of=x if epilogue else None)
        torch.cuda.synchronize()
        assert dx.untouched() and not dx.t[:2].any() and not dx.t[off[-1]:].any()
        for e in range(E):
            lo, hi = off[e], off[e + 1]
            want = dy[lo:hi].float() @ w[e].float()
            if epilogue:
                want = want * (x[lo:hi] > 0)
            assert torch.equal(dx.t[lo:hi], want.to(TORCH[out])), (e, epilogue, out)
