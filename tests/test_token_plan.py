"""The plan of the token-model operators' products (tile and slices), asked on
the CPU of the header that holds it: that the GPU tests' sizes reach every kernel."""
import os
import subprocess

import pytest

from tests.token_shapes import TILES, products

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <stdio.h>
#include "paper_1912_11554_amd/csrc/token.h"
using namespace nuts::token;
int main()
{
    long long M, N, K;
    int f32, staged, gated, terms, sets;
    while (scanf("%lld %lld %lld %d %d %d %d %d", &M, &N, &K, &f32, &staged, &gated, &terms, &sets) == 8) {
        Product p{};
        p.M = M, p.N = N, p.K = K, p.dtype = f32 ? NUTS_F32 : NUTS_BF16;
        p.staged = staged, p.gated = gated, p.nterms = terms, p.sets = sets;
        const Plan plan = plan_product(p, 256);
        printf("%d %d %d\n", plan.tile, plan.slices, (int)few_rows(M, N, K));
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    at = tmp_path_factory.mktemp("plan")
    src, exe = at / "plan.cpp", at / "plan"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", ROOT, "-I", rocm + "/include", str(src), "-o",
                    str(exe)], check=True, capture_output=True, text=True)

    def ask(asked):
        lines = "\n".join(" ".join(str(int(v)) for v in q) for q in asked)
        out = subprocess.run([str(exe)], input=lines, check=True, capture_output=True, text=True).stdout.split("\n")
        return [tuple(map(int, line.split())) for line in out if line]

    return ask


@pytest.mark.parametrize("case", TILES, ids=lambda c: "-".join(map(str, c[:5])))
def test_sizes_reach_their_tiles(plan, case):
    kind, dtype, M, N, K, want = case
    got = plan(products(kind, dtype, M, N, K))
    assert [(tile, slices > 1) for tile, slices, _ in got] == list(want)
    assert not any(few for _, _, few in got[:1])


def test_every_kernel_of_the_products_is_reached():
    # (staged, tile, operands' order, type): with the small sizes of the other tests, which are 64 x 64
    seen = set()
    for kind, dtype, M, N, K, want in TILES:
        for order, p, (tile, _) in zip(("forward", "dx", "dw"), products(kind, dtype, M, N, K), want):
            seen.add((p[4], tile, kind + " " + order if order == "forward" else order, dtype))
    for order in ("linear forward", "gated forward", "dx", "dw"):
        assert {(False, 256, order, "bfloat16"), (False, 128, order, "bfloat16"), (True, 128, order, "bfloat16"),
                (True, 128, order, "float32")} <= seen
