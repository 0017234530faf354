"""Products with low-rank adapters on every way that the library has for them, against plain sums in 64 bits (tolerances: test_gpu_adapters.py)."""
import pytest
import torch

import paper_2210_12415_amd as alt
from adapters_ways import WAYS
from rows_util import TORCH, matrix, normal, replayed, ws
from test_gpu_adapters import check, requests

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    return alt.Handle()


IDS = ["-".join(map(str, w)).replace(" ", "_") for w in WAYS]


@pytest.mark.parametrize("case", WAYS, ids=IDS)
def test_adapters_on_every_way(h, case):
    way, kernel, dtype, M, N, K, G, r = case
    check(h, M, N, K, G, r, requests(M, G), dtype, out=alt.F32)
    check(h, M, N, K, G, r, requests(M, G, 1, (1, 3)), dtype, relu=True)


@pytest.mark.parametrize("case", WAYS, ids=IDS)
def test_adapters_on_every_way_in_rows_apart(h, case):
    """Rows with gaps; whole chunks stay whole chunks."""
    way, kernel, dtype, M, N, K, G, r = case
    check(h, M, N, K, G, r, requests(M, G, 2, (1, 200)), dtype, strides=(K + 16, K + 32, N + 8))


@pytest.mark.parametrize("case", [w for w in WAYS if w[0] != "few"], ids=[i for w, i in zip(WAYS, IDS) if w[0] != "few"])
def test_adapters_on_every_way_give_the_same_bits_from_graphs(h, case):
    """A call captured on another stream, and eager calls between its replays."""
    way, kernel, dtype, M, N, K, G, r = case
    t = TORCH[dtype]
    x, w = matrix(normal(1, M, K), t), matrix(normal(2, N, K, std=K ** -0.5), t)
    a, b = matrix(normal(3, G * r, K, std=K ** -0.5), t).view(G, r, K), matrix(normal(4, G * N, r), t).view(G, N, r)
    ids = torch.tensor(requests(M, G, 3), dtype=torch.int32, device="cuda")
    d = alt.adapters_desc(M, N, K, G, r, in_dtype=dtype, out_dtype=dtype)
    y, space = torch.empty(M, N, dtype=t, device="cuda"), ws(h.gemm_adapters_workspace_size(d))
    replayed(lambda: h.gemm_adapters(d, x, w, ids, a, b, y, **space), [y], lambda: y.fill_(3))
