"""Which way the product in 8 bits takes (host arithmetic, compiled on its own: no GPU), and that the tests run every kernel that the ways lead to.

A size takes one of: workgroups of 16 or 32 rows whose waves share the columns, by 16 to 128 columns of the result; tiles of 64, 128 or 256 through LDS in two or four stages; tiles of
128 for parts of the columns, whose sums a second kernel adds and finishes.
"""
import math
import os
import random
import subprocess

import pytest
import torch

import test_block8 as block8

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DTYPES = [torch.float32, torch.bfloat16, torch.float8_e4m3fn]       # by their numbers in the descriptor
ACTS = ["none", "gelu", "swiglu"]
F32, BF16, E4M3 = range(3)
NONE, GELU, SWIGLU = range(3)

PROGRAM = r"""
#include <cstdio>
#include "matmul8_plan.h"
// M N K dtype act cus -> rows columns splits stages
int main() {
  long long M;
  int N, K, dtype, act, cus;
  while (std::scanf("%lld %d %d %d %d %d", &M, &N, &K, &dtype, &act, &cus) == 6) {
    const svdc::MatmulPlan plan = svdc::matmul8_plan({M, N, K, dtype, act, N}, cus);
    std::printf("%d %d %d %d\n", plan.rows, plan.columns, plan.splits, plan.stages);
  }
}
"""


@pytest.fixture(scope="module")
def ways(tmp_path_factory):
    d = tmp_path_factory.mktemp("ways")
    src, exe = str(d / "ways.cpp"), str(d / "ways")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2601_07396_amd", "csrc"), "-o", exe, src], check=True)

    def run(products, cus=256):
        text = "\n".join(" ".join(str(int(x)) for x in (*p, cus)) for p in products)
        out = subprocess.run([exe], input=text, stdout=subprocess.PIPE, text=True, check=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    return run


# Beside the sizes of test_block8.py: those that nothing there takes the way of
FURTHER = [
    (272, 925, 743, F32, GELU), (3, 8427, 276, BF16, GELU), (24, 2375, 278, F32, GELU), (18, 2144, 328, BF16, GELU), (130, 946, 423, F32, GELU), (290, 968, 829, F32, GELU),
    (1637, 133, 679, BF16, GELU), (4, 3, 15955, F32, GELU), (11432, 130, 271, F32, GELU), (65, 17630, 262, BF16, GELU), (16431, 3, 268, E4M3, NONE), (2740, 4361, 551, BF16, GELU),
    (19770, 598, 553, E4M3, NONE)]


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,dtype,act", FURTHER)
def test_matmul8_further_ways(M, N, K, dtype, act):
    block8.check_product(M, N, K, DTYPES[dtype], ACTS[act], with_bias=N % 2 == 1, seed=N, planted=M % 2 == 0, ldo_pad=5 if M % 3 == 0 else 0)


def products_of_tests():
    """The sizes of the GPU tests, from their parameters."""
    out = list(FURTHER)
    for test in (block8.test_matmul8, block8.test_matmul8_larger, block8.test_matmul8_nan_stays_in_its_row, block8.test_matmul8_every_way, block8.test_matmul8_few_tiles_of_long_sums):
        cases = [{"act": "gelu"}]
        for mark in test.pytestmark:
            if mark.name == "parametrize":
                names, values = mark.args[0].split(","), mark.args[1]
                cases = [{**c, **dict(zip(names, v if len(names) > 1 else (v,)))} for c in cases for v in values]
        out += [(c["M"], c["N"], c["K"], DTYPES.index(c["dtype"]), ACTS.index(c["act"])) for c in cases]
    return out


def kernels(product, way):
    """What is launched, as far as it is compiled or branches apart."""
    *_, dtype, act = product
    rows, columns, splits, stages = way
    if rows <= 32:
        return {("few rows", rows, columns, dtype, act)}
    if splits == 1:
        return {("tiles", rows, dtype, act, stages)}
    return {("sums", dtype == F32, stages), ("parts", dtype == F32, splits), ("finish", dtype, act)}


def all_kernels():
    few = {("few rows", rows, columns, dtype, act) for rows in (16, 32) for dtype in (F32, BF16) for act in range(3) for columns in (16, 32, 64) if act != SWIGLU or columns < 64}
    few |= {("few rows", 16, 128, E4M3, act) for act in (NONE, GELU)}
    tiles = {("tiles", rows, F32, act, 2) for rows in (64, 128) for act in range(3)}
    tiles |= {("tiles", rows, BF16, act, stages) for rows in (64, 128) for act in range(3) for stages in (2, 4)} | {("tiles", 256, BF16, act, 2) for act in range(3)}
    tiles |= {("tiles", rows, E4M3, act, stages) for rows in (64, 128) for act in range(3) for stages in (2, 4) if act != SWIGLU or stages == 2}
    tiles |= {("tiles", 256, E4M3, act, 2) for act in range(3)}
    parts = {("sums", True, 2), ("sums", False, 2), ("sums", False, 4)} | {("parts", exact, n) for exact in (True, False) for n in (2, 4, 8, 16)}
    return few | tiles | parts | {("finish", dtype, act) for dtype in range(3) for act in range(3)}


def test_every_kernel_is_reached_and_tested(ways):
    """What ordinary sizes reach is all that there is, and all of it is run by a test of this file or of test_block8.py."""
    rng = random.Random(5)

    def size():
        return round(math.exp(rng.uniform(0, math.log(20000))))

    some = [(size(), size(), size(), rng.randrange(3), rng.randrange(3)) for _ in range(200000)]
    reached = set().union(*map(kernels, some, ways(some)))
    assert reached == all_kernels()
    products = products_of_tests()
    assert all_kernels() - set().union(*map(kernels, products, ways(products))) == set()
