"""What the calls around the layers' products refuse, before any device work, and how their arguments are marshalled."""
import pytest

import paper_2210_12415_amd as alt

INVALID, SHAPE, UNSUPPORTED, WORKSPACE, HIP = 1, 3, 4, 5, 6

# call -> (descriptor, its arguments, the buffers, those that may be null, and the workspace's size call)
DESC = {"norm": (alt.norm_desc, dict(rows=4, cols=64)), "route": (alt.route_desc, dict(tokens=4, experts=16, top_k=2)),
        "exchange": (alt.exchange_desc, dict(tokens=4, top_k=2, rows=8, cols=64)), "adapters": (alt.adapters_desc, dict(M=4, N=32, K=64, adapters=2, rank=8, epilogue=alt.EPI_BIAS))}
CALLS = {"layer_norm": ("norm", ("x", "y", "gamma", "beta", "mean", "rstd"), ("gamma", "beta", "mean", "rstd"), False),
         "layer_norm_grad": ("norm", ("dy", "x", "mean", "rstd", "dx", "gamma", "dgamma", "dbeta"), ("gamma", "dgamma", "dbeta"), True),
         "route": ("route", ("logits", "experts", "weights", "rows", "offsets", "bias"), ("bias",), True),
         "route_grad": ("route", ("logits", "experts", "dweights", "dlogits"), (), False),
         "dispatch_rows": ("exchange", ("x", "rows", "y"), (), False),
         "combine_rows": ("exchange", ("x", "rows", "y", "weights"), ("weights",), False),
         "combine_rows_grad": ("exchange", ("dy", "x", "rows", "weights", "dx", "dweights"), ("weights", "dweights"), False),
         "gemm_adapters": ("adapters", ("x", "w", "adapter", "a", "b", "y", "scale", "bias"), ("scale",), True)}


@pytest.fixture(scope="module")
def h():
    return alt.Handle()


def desc(kind, **change):
    make, a = DESC[kind]
    return make(**dict(a, **change))


def arguments(name, **change):
    kind, buffers, _, space = CALLS[name]
    a = dict({b: 4096 for b in buffers}, stream=0)
    if space:
        a.update(workspace=4096, ws_bytes=1 << 30)
    a.update(change)
    return a


def refused(call):
    with pytest.raises(alt.AltError) as e:
        call()
    assert str(e.value).count(":") >= 1               # says what
    return e.value.status


SIZES = {"norm": [(dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(in_dtype=alt.I8), INVALID), (dict(out_dtype=7), INVALID), (dict(eps=-1e-9), INVALID),
                  (dict(eps=float("nan")), INVALID), (dict(x_stride=-1), INVALID), (dict(x_stride=63), SHAPE), (dict(y_stride=63), SHAPE), (dict(rows=1 << 31), UNSUPPORTED),
                  (dict(cols=1 << 25), UNSUPPORTED), (dict(x_stride=1 << 32), UNSUPPORTED)],
         "route": [(dict(tokens=-1), INVALID), (dict(experts=0), INVALID), (dict(top_k=0), INVALID), (dict(dtype=alt.I8), INVALID), (dict(score=2), INVALID),
                   (dict(renormalize=2), INVALID), (dict(groups=0), INVALID), (dict(top_groups=0), INVALID), (dict(top_groups=2), INVALID), (dict(group_best=3), INVALID),
                   (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(stride=-1), INVALID), (dict(stride=15), SHAPE), (dict(groups=3, top_groups=3), SHAPE),
                   (dict(top_k=17), SHAPE), (dict(groups=8, top_groups=1, top_k=3), SHAPE), (dict(experts=1025), UNSUPPORTED), (dict(experts=64, top_k=33), UNSUPPORTED),
                   (dict(tokens=1 << 30), UNSUPPORTED), (dict(stride=1 << 32), UNSUPPORTED)],
         "exchange": [(dict(tokens=-1), INVALID), (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(top_k=0), INVALID), (dict(dtype=alt.I8), INVALID),
                      (dict(token_stride=-1), INVALID), (dict(row_stride=63), SHAPE), (dict(token_stride=63), SHAPE), (dict(top_k=33), UNSUPPORTED), (dict(tokens=1 << 30), UNSUPPORTED),
                      (dict(rows=1 << 31), UNSUPPORTED), (dict(cols=1 << 25), UNSUPPORTED), (dict(row_stride=1 << 32), UNSUPPORTED)],
         "adapters": [(dict(M=-1), INVALID), (dict(N=0), INVALID), (dict(K=0), INVALID), (dict(adapters=0), INVALID), (dict(rank=0), INVALID), (dict(in_dtype=alt.I8), INVALID),
                      (dict(out_dtype=alt.I8), INVALID), (dict(epilogue=4), INVALID), (dict(lda=-1), INVALID), (dict(lda=63), SHAPE), (dict(ldb=63), SHAPE), (dict(ldc=31), SHAPE),
                      (dict(in_dtype=alt.F32), UNSUPPORTED), (dict(rank=513), UNSUPPORTED), (dict(adapters=1 << 21), UNSUPPORTED), (dict(N=1 << 25), UNSUPPORTED),
                      (dict(M=1 << 31), UNSUPPORTED), (dict(lda=1 << 23), UNSUPPORTED)]}


@pytest.mark.parametrize("name,change,status", [(n, c, s) for n in CALLS for c, s in SIZES[CALLS[n][0]]])
def test_refuses_descriptors(h, name, change, status):
    d = desc(CALLS[name][0], **change)
    assert refused(lambda: getattr(h, name)(d, **arguments(name))) == status
    if CALLS[name][3]:
        assert refused(lambda: getattr(h, name + "_workspace_size")(d)) == status


@pytest.mark.parametrize("name,buffer", [(n, b) for n in CALLS for b in CALLS[n][1]])
def test_refuses_buffers(h, name, buffer):
    d = desc(CALLS[name][0])
    if buffer not in CALLS[name][2]:
        assert refused(lambda: getattr(h, name)(d, **arguments(name, **{buffer: None}))) == INVALID
    assert refused(lambda: getattr(h, name)(d, **arguments(name, **{buffer: 4097}))) == INVALID


@pytest.mark.parametrize("name", [n for n in CALLS if CALLS[n][3]])
def test_refuses_workspaces(h, name):
    d = desc(CALLS[name][0])
    need = getattr(h, name + "_workspace_size")(d)
    assert need > 0
    assert refused(lambda: getattr(h, name)(d, **arguments(name, ws_bytes=need - 1))) == WORKSPACE
    assert refused(lambda: getattr(h, name)(d, **arguments(name, workspace=None))) == WORKSPACE


def test_workspaces_hold_what_is_counted_in_64_bits(h):
    assert h.gemm_adapters_workspace_size(desc("adapters", M=1 << 29, rank=512)) >= (1 << 29) * 512 * 4
    assert h.layer_norm_grad_workspace_size(desc("norm", rows=1 << 29, cols=1 << 24)) >= 2 * 4 << 24


@pytest.mark.parametrize("name", sorted(CALLS))
def test_calls_without_a_gpu_fail_loudly(h, name):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert refused(lambda: getattr(h, name)(desc(CALLS[name][0]), **arguments(name))) == HIP


class Tensor:
    def data_ptr(self):
        return 4096


@pytest.mark.parametrize("name", sorted(CALLS))
def test_native_and_ctypes_calls_agree(h, name, monkeypatch):
    """Every argument that the native marshalling takes, and some that it leaves to ctypes, end alike (here, without a GPU, in the library's status)."""
    import os

    import numpy as np

    from paper_2210_12415_amd import binding
    if binding._native is None or os.path.exists("/dev/kfd"):
        pytest.skip("needs the native module, and no GPU: the addresses are of no buffer")
    first = CALLS[name][1][0]
    base = arguments(name, d=desc(CALLS[name][0]))
    forms = [dict(d=None), {first: Tensor()}, {first: None}, {first: "text"}, {first: np.int64(4096)}, {first: 4097}, dict(stream="text"), dict(stream=np.int64(0))]
    if CALLS[name][3]:
        forms += [dict(workspace=Tensor()), dict(ws_bytes=np.int64(8)), dict(ws_bytes=None), dict(ws_bytes=8)]

    def outcome(kw):
        try:
            return getattr(h, name)(**kw)
        except Exception as e:
            return type(e), str(e)
    quick, taken = "_quick_" + name, []
    native = getattr(binding, quick)
    for form in [{}] + forms:
        kw = dict(base, **form)
        monkeypatch.setattr(binding, quick, lambda *a: taken.append(native(*a)) or taken[-1])
        one = outcome(kw)
        monkeypatch.setattr(binding, quick, binding._not_taken)
        assert one == outcome(kw), form
    assert any(t is not None for t in taken) and any(t is None for t in taken)
