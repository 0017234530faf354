"""Layer norm and its gradients where every thread has several rows one after another (the next one on its way while one is reduced, sums in one of two places in
turn), against the formulas in 64 bits (tolerances: test_gpu_norm.py)."""
import pytest
import torch

import paper_2210_12415_amd as alt
from rows_util import TORCH, matrix
from test_gpu_norm import TYPES, check, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    return alt.Handle()


# (256 compute units: forward 8192 rows at once up to 1024 columns, 2048 up to 4096, 1024 up to 8192, 512 up to 16384; gradients 2048 up to 512 columns, 1024 up to 1024,
# 512 up to 2048, 256 beyond; more than 16384 columns: 64 shares of the columns' sums)
SHAPES = [(17000, 100), (8300, 500), (8300, 513), (8300, 1000), (2100, 1025), (4500, 1500), (2100, 2050), (2100, 4096), (1100, 4200), (1100, 8192), (600, 8200), (530, 12345), (520, 16384), (70, 16385),
          (200, 20011)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("types", TYPES)
def test_norm_of_several_rows_to_a_thread(h, rows, cols, types):
    x, gamma, beta, dy = inputs(rows, cols)
    check(h, matrix(x, TORCH[types[0]]), gamma.cuda(), beta.cuda(), matrix(dy, TORCH[types[1]]), types)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,cols,ldx,ldy", [(17000, 63, 65, 71), (8300, 700, 701, 703), (2100, 2050, 2051, 2053), (2100, 1501, 1503, 1504), (1100, 4200, 4201, 4204), (520, 16383, 16385, 16387)])
def test_norm_of_several_rows_to_a_thread_at_any_alignment(h, rows, cols, ldx, ldy, types):
    x, gamma, beta, dy = inputs(rows, cols, 9)
    check(h, matrix(x, TORCH[types[0]], ldx, 1), gamma.cuda(), beta.cuda(), matrix(dy, TORCH[types[1]], ldy, 1), types, strides=(ldx, ldy), offset=1)


def test_norm_of_several_rows_special_values_stay_in_theirs(h):
    """A row of NaN and one of infinities among those of every thread."""
    both = (alt.BF16, alt.BF16)
    for rows, cols in ((17000, 300), (4500, 1500), (2500, 5000), (1100, 9000)):
        x, gamma, beta, dy = inputs(rows, cols, 2)
        x, dy, gamma, beta = matrix(x, torch.bfloat16), matrix(dy, torch.bfloat16), gamma.cuda(), beta.cuda()
        d = alt.norm_desc(rows, cols)

        def run(x):
            y, mean, rstd, dx = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
            h.layer_norm(d, x, y, gamma=gamma, beta=beta, mean=mean, rstd=rstd)
            h.layer_norm_grad(d, dy, x, mean, rstd, dx, gamma=gamma)
            torch.cuda.synchronize()
            return y, mean, rstd, dx
        bad = x.clone()
        lost = torch.zeros(rows, dtype=torch.bool, device="cuda")
        lost[5::7] = True
        bad[5::14, cols - 1], bad[12::14, 3] = float("nan"), float("inf")
        clean, got = run(x), run(bad)
        assert torch.isnan(got[0][lost].float()).all() and torch.isnan(got[3][lost].float()).all()
        for a, b in zip(got, clean):
            assert torch.equal(a[~lost], b[~lost])
