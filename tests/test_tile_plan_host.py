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

# M, K, N of gradients whose two products share a launch: kind, whether dx's and dw's sums are in parts
JOINT = {
    ("256x256", False, False): (1564, 3985, 1433), ("256x128", False, False): (516, 3841, 661), ("256x128", False, True): (5095, 1812, 65),
    ("256x128", True, False): (95, 1914, 4998), ("256x128", True, True): (2960, 133, 5557), ("128x128", False, False): (208, 3271, 324),
    ("128x128", False, True): (5048, 911, 8), ("128x128", True, False): (8, 827, 5601), ("128x128", True, True): (3151, 69, 2639),
    ("128x128 two", False, False): (395, 3611, 575), ("128x128 two", False, True): (1251, 2399, 67), ("128x128 two", True, False): (65, 1811, 1705),
    ("128x64", False, False): (8, 2638, 464), ("128x64", False, True): (4342, 263, 8), ("128x64", True, False): (8, 391, 3025),
    ("128x64", True, True): (1235, 1, 3370), ("64x64", False, False): (8, 1, 65), ("64x64", False, True): (782, 1, 8), ("64x64", True, False): (8, 1, 770),
    ("64x64", True, True): (911, 1, 1415), ("64x64 six", False, False): (8, 1, 8), ("64x64 six", False, True): (1127, 2719, 8),
    ("64x64 six", True, False): (8, 3120, 970),
}

# ... and of gradients whose products are two launches: dx's kind, in parts or not, dw's
APART = {
    ("256x256", False, "128x128", True): (4308, 3808, 206), ("128x128", True, "256x256", False): (257, 2654, 4802), ("256x128", False, "128x128", True): (3853, 1757, 453),
    ("128x64", False, "128x128", False): (1523, 1127, 2112), ("128x128", True, "128x128 two", False): (68, 3518, 5940), ("128x128 two", False, "128x64", True): (5622, 2820, 72),
    ("64x64", True, "64x64 six", False): (8, 1852, 2491), ("64x64 six", False, "64x64", True): (4575, 1048, 8), ("64x64", True, "128x128 two", False): (8, 1302, 4864),
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


def test_gradients_take_every_kind_of_tile_in_one_launch(plan):
    keys = list(JOINT)
    for key, (_, joint, k0, s0, k1, s1) in zip(keys, plan([JOINT[k] for k in keys])):
        assert joint and (KINDS[k0], s0 > 1, s1 > 1) == key and k0 == k1
    assert {k[0] for k in keys} == set(KINDS)


def test_gradients_in_two_launches(plan):
    keys = list(APART)
    for key, (_, joint, k0, s0, k1, s1) in zip(keys, plan([APART[k] for k in keys])):
        assert not joint and (KINDS[k0], s0 > 1, KINDS[k1], s1 > 1) == key
