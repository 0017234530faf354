"""Matrices with guards, and comparisons, for the tests of the calls around the layers' products."""
import numpy as np
import torch

import paper_2210_12415_amd as alt

TORCH = {alt.F32: torch.float32, alt.BF16: torch.bfloat16}
EPS = 2.0 ** -24                          # of one rounding to fp32, relative to the value
HALF = {alt.F32: 2.0 ** -24, alt.BF16: 2.0 ** -8}
TINY = {alt.F32: 2.0 ** -148, alt.BF16: 2.0 ** -132}     # where values are too small for a relative rounding


class Guarded:
    """A device matrix with unused columns and guards around it, all holding a pattern; `offset` elements into its buffer."""

    def __init__(self, rows, cols, dtype, stride=0, offset=0, device="cuda"):
        self.stride = stride or cols
        n = rows * self.stride
        self.whole = torch.full((n + 256 + offset,), 77, dtype=dtype, device=device)
        self.at = self.whole[128 + offset:128 + offset + n]
        self.cols, self.lo = cols, 128 + offset
        self.t = self.at.view(rows, self.stride)[:, :cols]

    def data_ptr(self):
        return self.at.data_ptr()

    def untouched(self):
        n = self.at.numel()
        return bool((self.whole[:self.lo] == 77).all()) and bool((self.whole[self.lo + n:] == 77).all()) and bool((self.at.view(-1, self.stride)[:, self.cols:] == 77).all())


def matrix(values, dtype, stride=0, offset=0):
    """A device matrix with `values` in rows `stride` apart (what lies between them is NaN), `offset` elements into its buffer."""
    values = torch.as_tensor(values)
    rows, cols = values.shape
    stride = stride or cols
    buf = torch.full((rows * stride + offset,), float("nan"), dtype=dtype, device="cuda")
    view = buf[offset:].view(rows, stride)[:, :cols]
    view.copy_(values.to(dtype))
    return view


def normal(seed, *shape, std=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g) * std + mean


def f64(t):
    return t.detach().cpu().double().numpy()


def ws(size, offset=0):
    """A workspace as the calls take it, `offset` bytes into its buffer and full of NaN."""
    if not size:
        return dict(workspace=None, ws_bytes=0)
    return dict(workspace=torch.full((size + offset,), 255, dtype=torch.uint8, device="cuda")[offset:], ws_bytes=size)


def close(got, want, tol, what=""):
    got, want = f64(got), np.asarray(want)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~(np.abs(got - want) <= tol) & (got != want) & ~(np.isnan(got) & np.isnan(want))
    if bad.any():
        at = tuple(np.argwhere(bad)[0])
        raise AssertionError("%s: %d of %d off, first at %s: %r for %r, allowed %r" % (what, bad.sum(), bad.size, at, got[at], want[at], np.broadcast_to(tol, got.shape)[at]))


def equal(got, want, what=""):
    got, want = got.cpu().numpy(), np.asarray(want)
    assert got.shape == want.shape and np.array_equal(got, want), "%s: %s differ" % (what, np.argwhere(got != want)[:4].tolist() if got.shape == want.shape else (got.shape, want.shape))


def replayed(run, outputs, reset, times=3):
    """Captures `run` and replays it, with eager work and synchronisation between the replays; every replay has to give what the eager call gave."""
    run()
    torch.cuda.synchronize()
    want = [o.clone() for o in outputs]
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    for _ in range(times):
        reset()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for o, w in zip(outputs, want):
            assert torch.equal(o.view(torch.uint8) if o.is_contiguous() else o, w.view(torch.uint8) if o.is_contiguous() else w)
        run()
