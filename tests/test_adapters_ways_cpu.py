"""Which way a product with adapters takes, by the library's own rule: the sizes of adapters_ways.py reach every one, so that a constant that moves empties no test."""
import os
import subprocess

import pytest

import paper_2210_12415_amd as alt
from adapters_ways import WAYS

CSRC = os.path.join(os.path.dirname(alt.__file__), "csrc")
OBJECT = os.path.join(CSRC, "_build", "adapters.hip.o")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

PROGRAM = r'''
#include "adapters.h"
int main()
{
    long dtype, M, N, K, G, r;
    while (scanf("%ld %ld %ld %ld %ld %ld", &dtype, &M, &N, &K, &G, &r) == 6) {
        const int es = dtype == ALT_F32 ? 4 : 2;
        alt::GroupedParams p{};
        p.rows = (int)M; p.cols = (int)N; p.red = (int)K;
        p.lda = p.ldb = K * es;
        p.groups = 1; p.places = 256;
        alt::AdapterParams q{};
        q.rows = p.rows; q.cols = p.cols; q.K = p.red;
        q.rank = (int)r; q.adapters = (int)G; q.places = p.places;
        alt::adapters_plan((int)dtype, p, q);
        alt::GrpTime t;
        printf("%s %d %d %d %d %zu %.0f %.0f\n", q.few ? "few" : q.beside ? "beside" : "fused", alt::grp_choose<alt::kForward>(p, es, &t), q.few_cols, q.base_slices, q.slices,
               alt::adapters_inner_bytes((int)dtype, q), alt::grp_tiles<alt::kForward>(p, 64, 64), alt::grp_tiles<alt::kForward>(p, 128, 128));
    }
}
'''


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if not os.path.exists(OBJECT) or not os.path.exists(HIPCC):
        pytest.skip("no compiled kernels, or no compiler")
    folder = tmp_path_factory.mktemp("ways")
    with open(folder / "ways.cpp", "w") as f:
        f.write(PROGRAM)
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-x", "hip", "--cuda-host-only", "-w", "-I" + CSRC, "-c", "ways.cpp", "-o", "ways.o"], cwd=folder, check=True)
    subprocess.run([HIPCC, "ways.o", OBJECT, "-o", "ways"], cwd=folder, check=True)
    lines = "\n".join(" ".join(map(str, w[2:])) for w in WAYS)
    return subprocess.run(["./ways"], cwd=folder, input=lines, check=True, capture_output=True, text=True).stdout.splitlines()


@pytest.mark.parametrize("i", range(len(WAYS)), ids=lambda i: "-".join(map(str, WAYS[i])).replace(" ", "_"))
def test_the_way_of(plans, i):
    way, kernel, dtype, M, N, K, G, r = WAYS[i]
    got, tiles, few_cols, base_slices, slices, inner, n64, n128 = plans[i].split()
    assert got == way
    d = alt.adapters_desc(M, N, K, G, r, in_dtype=dtype, out_dtype=alt.F32)
    base = 0 if way == "fused" else int(base_slices) * M * N * 4
    packed = alt.Handle().gemm_adapters_workspace_size(d) > int(inner) + (base + 15) // 16 * 16 + 16
    if way == "few":
        assert kernel == "%s %s %s" % (few_cols, base_slices, slices) and not packed
    elif packed:
        assert kernel == "packed"
    elif K * (4 if dtype == alt.F32 else 2) % 16 == 0:
        assert kernel == ("ring" if dtype == alt.F32 else ["deep", "shallow", "half", "middle", "large"][int(tiles)])
    else:
        assert kernel == ("any 128" if dtype == alt.BF16 and float(n128) >= 128 else "any 64" if float(n64) <= 512 else "any 64 many")


def test_every_way_is_there():
    """All ways, and each with every kind of product that it runs."""
    ways = {}
    for way, kernel, dtype, *_ in WAYS:
        ways.setdefault((way, dtype), set()).add(kernel)
    assert {("few", alt.BF16), ("few", alt.F32), ("beside", alt.BF16), ("beside", alt.F32), ("fused", alt.BF16), ("fused", alt.F32)} == set(ways)
    assert ways["fused", alt.BF16] == {"deep", "shallow", "half", "middle", "large", "any 128", "any 64", "packed"}
    assert ways["fused", alt.F32] == {"ring", "any 64", "any 64 many"}
    assert ways["beside", alt.BF16] >= {"deep", "half", "middle", "large", "any 128", "any 64", "packed"}
