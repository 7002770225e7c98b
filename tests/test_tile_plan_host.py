"""Which tiles the dense products of the GPU tests take on 256 compute units (host code only: tile_plan.hpp, compiled for the CPU).  The sizes here are
those that tests/test_gpu_tile_kinds.py runs: a planner that is fitted anew and leaves a kind of tile without a test shows up here."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2203_04071_amd", "csrc")

KINDS = ("256x256", "256x128", "128x128", "128x128 two", "128x64", "64x64", "64x64 six")
STAGE = {"256x256": 64, "256x128": 128, "128x128": 128, "128x128 two": 64, "128x64": 128, "64x64": 128, "64x64 six": 64}       # bytes of a row

# M, K, N of exact products: last tiles that are not whole in both directions; rows of whole stages and not, of fewer stages than a tile has buffers and
# of more
PRODUCTS = {
    "256x256": [(3600, 784, 3423), (4558, 832, 2859)],
    "256x128": [(2782, 928, 2859), (1799, 1280, 3771)],
    "128x128": [(580, 1456, 3322), (4718, 1536, 389)],
    "128x128 two": [(1801, 16, 3332), (1805, 64, 3357), (1409, 80, 4260), (1249, 128, 4865), (4911, 144, 1229), (4938, 336, 1229), (1306, 384, 4711)],
    "128x64": [(329, 528, 4851), (338, 656, 4557), (3185, 640, 516)],
    "64x64": [(70, 400, 1437), (65, 512, 1507), (68, 528, 1526), (66, 768, 1607)],
    "64x64 six": [(67, 16, 1452), (66, 80, 1464), (65, 128, 1458), (70, 144, 1426), (67, 336, 1443), (65, 384, 1603)],
}

PROGRAM = r'''
#include <cstdio>
#include "tile_plan.hpp"
using namespace adapt_api;
int main() {
    long long M, K, N;
    while (std::scanf("%lld %lld %lld", &M, &K, &N) == 3) {
        const TilePlan t = tile_plan(M, N, K, 256, 1);
        // pieces of dy s: two fp16 numbers an element, in whole stages of 64
        const long long I[2] = {M, N}, J[2] = {K, K}, Kb[2] = {4 * ((N + 63) / 64 * 64), 4 * ((M + 63) / 64 * 64)};
        const TilePairPlan p = tile_pair_plan(I, J, Kb, 256);
        std::printf("%d %d %d %d %d %d\n", (int)t.kind, (int)p.joint, (int)p.plan[0].kind, p.plan[0].split, (int)p.plan[1].kind, p.plan[1].split);
    }
    return 0;
}
'''


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """(kind of the exact product, joint, dx's kind, parts, dw's kind, parts) for every M, K, N"""
    d = tmp_path_factory.mktemp("tiles")
    src, exe = d / "plan.cpp", d / "plan"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", CSRC, str(src), "-o", str(exe)], check=True, timeout=120)

    def call(sizes):
        out = subprocess.run([str(exe)], input="\n".join("%d %d %d" % s for s in sizes), check=True, capture_output=True, text=True, timeout=60).stdout
        rows = [tuple(int(v) for v in line.split()) for line in out.splitlines()]
        assert len(rows) == len(sizes)
        return rows
    return call


def test_products_take_every_kind_of_tile(plan):
    assert set(PRODUCTS) == set(KINDS)
    for kind, sizes in PRODUCTS.items():
        assert [KINDS[row[0]] for row in plan(sizes)] == [kind] * len(sizes), kind
        for M, K, N in sizes:
            assert K % 16 == 0 and 5 * -(-N // 16) * -(-M // 64) >= 900         # (neither ragged rows nor the kernel without LDS tiles)
        assert {K % STAGE[kind] == 0 for _, K, _ in sizes} == {False, True}     # a last stage that is whole, one that is not
        tm, tn = (int(v) for v in kind.split()[0].split("x"))
        assert any(M % tm and N % tn for M, _, N in sizes)
