"""What the 8-bit and the expert layers' entry points refuse, before any device work."""
import pytest

import paper_2210_12415_amd as alt

INVALID, SHAPE, UNSUPPORTED = 1, 3, 4


@pytest.fixture(scope="module")
def h():
    return alt.Handle()


def refused(call):
    with pytest.raises(alt.AltError) as e:
        call()
    assert str(e.value).count(":") >= 1               # says what
    return e.value.status


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(x_stride=-3), INVALID), (dict(q_stride=-1), INVALID), (dict(dtype=alt.I8), INVALID), (dict(dtype=9), INVALID),
    (dict(x_stride=63), SHAPE), (dict(q_stride=63), SHAPE), (dict(x=None), INVALID), (dict(q=None), INVALID), (dict(scale=None), INVALID), (dict(x=4097), INVALID),
    (dict(scale=4098), INVALID), (dict(rows=1 << 24), UNSUPPORTED), (dict(cols=1 << 31), UNSUPPORTED)])
def test_quantize_rows_refuses(h, change, status):
    a = dict(dtype=alt.BF16, rows=4, cols=64, x=4096, q=8192, scale=16384, stream=0)
    a.update(change)
    assert refused(lambda: h.quantize_rows(**a)) == status


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), INVALID), (dict(N=0), INVALID), (dict(K=0), INVALID), (dict(out_dtype=alt.I8), INVALID), (dict(epilogue=4), INVALID), (dict(lda=-1), INVALID),
    (dict(lda=63), SHAPE), (dict(ldb=63), SHAPE), (dict(ldc=31), SHAPE), (dict(K=131073), UNSUPPORTED), (dict(M=1 << 31), UNSUPPORTED)])
def test_gemm_i8_refuses_descriptors(h, change, status):
    a = dict(M=4, N=32, K=64)
    a.update(change)
    d = alt.gemm_i8_desc(**a)
    assert refused(lambda: h.gemm_i8(d, 4096, 4096, 4096, 4096, 4096, bias=4096, stream=0)) == status
    assert refused(lambda: h.gemm_i8_workspace_size(d)) == status


@pytest.mark.parametrize("name", ["a", "a_scale", "b", "b_scale", "y", "bias"])
def test_gemm_i8_refuses_buffers(h, name):
    d = alt.gemm_i8_desc(4, 32, 64, epilogue=alt.EPI_BIAS)
    a = dict(a=4096, a_scale=4096, b=4096, b_scale=4096, y=4096, bias=4096, stream=0)
    assert refused(lambda: h.gemm_i8(d, **dict(a, **{name: None}))) == INVALID
    if name not in ("a", "b"):
        assert refused(lambda: h.gemm_i8(d, **dict(a, **{name: 4097}))) == INVALID


CALLS = {"gemm_grouped": dict(a=4096, b=4096, offsets=4096, y=4096, bias=4096), "gemm_grouped_dx": dict(dy=4096, b=4096, offsets=4096, dx=4096, relu_of=4096),
         "gemm_grouped_dw": dict(a=4096, dy=4096, offsets=4096, dw=4096, dbias=4096)}
EPILOGUE = {"gemm_grouped": alt.EPI_BIAS | alt.EPI_RELU, "gemm_grouped_dx": alt.EPI_RELU, "gemm_grouped_dw": alt.EPI_BIAS}


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), INVALID), (dict(groups=0), INVALID), (dict(N=0), INVALID), (dict(K=-4), INVALID), (dict(in_dtype=3), INVALID), (dict(out_dtype=alt.I8), INVALID),
    (dict(epilogue=8), INVALID), (dict(ldc=-1), INVALID), (dict(lda=63), SHAPE), (dict(ldb=63), SHAPE), (dict(ldc=31), SHAPE),
    (dict(in_dtype=alt.F32, out_dtype=alt.BF16), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED), (dict(groups=1 << 21), UNSUPPORTED)])
def test_grouped_refuses_descriptors(h, name, change, status):
    a = dict(rows=4, groups=2, N=32, K=64, epilogue=EPILOGUE[name])
    a.update(change)
    d = alt.grouped_desc(**a)
    assert refused(lambda: getattr(h, name)(d, stream=0, **CALLS[name])) == status
    assert refused(lambda: getattr(h, name + "_workspace_size")(d)) == status


@pytest.mark.parametrize("name,buffer", [(n, b) for n in sorted(CALLS) for b in CALLS[n]])
def test_grouped_refuses_buffers(h, name, buffer):
    d = alt.grouped_desc(4, 2, 32, 64, epilogue=EPILOGUE[name])
    assert refused(lambda: getattr(h, name)(d, stream=0, **dict(CALLS[name], **{buffer: None}))) == INVALID
    assert refused(lambda: getattr(h, name)(d, stream=0, **dict(CALLS[name], **{buffer: 4097}))) == INVALID


def test_grouped_refuses_what_an_8_bit_layer_lacks(h):
    d = alt.grouped_desc(4, 2, 32, 64, in_dtype=alt.I8)
    a = CALLS["gemm_grouped"]
    assert refused(lambda: h.gemm_grouped(d, a_scale=None, b_scale=4096, stream=0, **a)) == INVALID
    assert refused(lambda: h.gemm_grouped(d, a_scale=4096, b_scale=None, stream=0, **a)) == INVALID
    assert refused(lambda: h.gemm_grouped(d, a_scale=4098, b_scale=4096, stream=0, **a)) == INVALID
    for name in ("gemm_grouped_dx", "gemm_grouped_dw"):
        assert refused(lambda: getattr(h, name)(d, stream=0, **CALLS[name])) == UNSUPPORTED
    far = alt.grouped_desc(4, 2, 32, 131073, in_dtype=alt.I8)
    assert refused(lambda: h.gemm_grouped(far, a_scale=4096, b_scale=4096, stream=0, **a)) == UNSUPPORTED


def test_8_bit_reductions_end_where_their_sums_fit(h):
    """131071 products of -128 and -128 fit a 32-bit sum; 131072 are 2^31, which does not."""
    assert 131071 * 128 * 128 < 2 ** 31 <= 131072 * 128 * 128
    a = dict(CALLS["gemm_grouped"], a_scale=4096, b_scale=4096, stream=0)
    for K in (131071, 131072):
        one, layer = alt.gemm_i8_desc(4, 32, K), alt.grouped_desc(4, 2, 32, K, in_dtype=alt.I8)
        if K == 131071:
            h.gemm_i8_workspace_size(one), h.gemm_grouped_workspace_size(layer)
            continue
        assert refused(lambda: h.gemm_i8_workspace_size(one)) == UNSUPPORTED and refused(lambda: h.gemm_grouped_workspace_size(layer)) == UNSUPPORTED
        assert refused(lambda: h.gemm_i8(one, 4096, 4096, 4096, 4096, 4096, stream=0)) == UNSUPPORTED
        assert refused(lambda: h.gemm_grouped(layer, **a)) == UNSUPPORTED


def test_grouped_refuses_epilogues_of_the_other_direction(h):
    d = alt.grouped_desc(4, 2, 32, 64, epilogue=alt.EPI_BIAS)
    assert refused(lambda: h.gemm_grouped_dx(d, stream=0, **CALLS["gemm_grouped_dx"])) == INVALID
    d = alt.grouped_desc(4, 2, 32, 64, epilogue=alt.EPI_RELU)
    assert refused(lambda: h.gemm_grouped_dw(d, stream=0, **CALLS["gemm_grouped_dw"])) == INVALID


def test_calls_without_a_gpu_fail_loudly(h):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for name in CALLS:
        d = alt.grouped_desc(4, 2, 32, 64, epilogue=EPILOGUE[name])
        assert refused(lambda: getattr(h, name)(d, stream=0, **CALLS[name])) == 6
    assert refused(lambda: h.quantize_rows(alt.BF16, 4, 64, 4096, 8192, 16384, stream=0)) == 6
    assert refused(lambda: h.gemm_i8(alt.gemm_i8_desc(4, 32, 64), 4096, 4096, 4096, 4096, 4096, stream=0)) == 6


class Tensor:
    def __init__(self, at):
        self.at = at

    def data_ptr(self):
        return self.at


@pytest.mark.parametrize("name", ["quantize_rows", "gemm_i8"] + sorted(CALLS))
def test_native_and_ctypes_calls_agree(h, name, monkeypatch):
    """Every argument that the native marshalling takes, and some that it leaves to ctypes, end alike (here, without a GPU, in the library's status)."""
    import os

    import numpy as np

    from paper_2210_12415_amd import binding
    if binding._native is None or os.path.exists("/dev/kfd"):
        pytest.skip("needs the native module, and no GPU: the addresses are of no buffer")
    quick = {"quantize_rows": "_quick_quantize", "gemm_i8": "_quick_gemm_i8"}.get(name, name.replace("gemm", "_quick"))
    if name == "quantize_rows":
        base = dict(dtype=alt.BF16, rows=4, cols=64, x=4096, q=8192, scale=16384, stream=0)
        forms = [dict(rows=np.int64(4)), dict(rows=4.0), dict(rows=-1), dict(dtype=np.int32(1)), dict(dtype="1"), dict(x=Tensor(4096)), dict(x=None), dict(q="text"), dict(x_stride=1 << 63)]
    else:
        d = alt.gemm_i8_desc(4, 32, 64) if name == "gemm_i8" else alt.grouped_desc(4, 2, 32, 64, epilogue=EPILOGUE[name])
        base = dict(dict(a=4096, a_scale=4096, b=4096, b_scale=4096, y=4096) if name == "gemm_i8" else CALLS[name], d=d, stream=0)
        first = next(k for k in base)
        forms = [dict(d=None), {first: Tensor(4096)}, {first: None}, {first: "text"}, {first: np.int64(4096)}, dict(workspace=Tensor(4096), ws_bytes=64),
                 dict(ws_bytes=np.int64(8)), dict(ws_bytes=None), dict(stream="text")]

    def outcome(kw):
        try:
            return getattr(h, name)(**kw)
        except Exception as e:
            return type(e), str(e)
    native, taken = getattr(binding, quick), []
    for form in [{}] + forms:
        kw = dict(base, **form)
        monkeypatch.setattr(binding, quick, lambda *a: taken.append(native(*a)) or taken[-1])
        one = outcome(kw)
        monkeypatch.setattr(binding, quick, binding._not_taken)
        assert one == outcome(kw), form
    assert any(t is not None for t in taken) and any(t is None for t in taken)
