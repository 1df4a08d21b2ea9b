"""Products in 8 bits of very many rows: more tiles than one launch takes, within the documented 2^31 - 1 rows."""
import os
import random
import subprocess

import pytest
import torch

import paper_2601_07396_amd as svdc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16, E4M3 = range(3)

PROGRAM = r"""
#include <cstdio>
#include "matmul8_plan.h"
// M N K dtype act -> rows and splits of the way, workgroups of its largest launch and launches
int main() {
  long long M;
  int N, K, dtype, act;
  while (std::scanf("%lld %d %d %d %d", &M, &N, &K, &dtype, &act) == 5) {
    const bool gated = act == SVDC_ACT_SWIGLU, eight = dtype == SVDC_E4M3;
    const svdc::MatmulPlan plan = svdc::matmul8_plan({M, N, K, dtype, act, N}, 256);
    long long tiles = 0, launches = 1;
    if (plan.rows > 0 && plan.rows <= 32) {
      tiles = (M + plan.rows - 1) / plan.rows * ((N + plan.columns - 1) / plan.columns);
    } else if (plan.splits > 1) {
      tiles = (M + 127) / 128 * ((svdc::wide_of({M, N, K, dtype, act, N}) + 127) / 128) * plan.splits;
    } else if (plan.rows > 0) {
      const long long most = svdc::rows_of_launch(plan, N, gated, eight);
      const int columns = 64 * svdc::tile_width(plan.rows, gated, eight) / (gated ? 2 : 1);
      launches = most > 0 ? (M + most - 1) / most : 0;
      tiles = ((M < most ? M : most) + plan.rows - 1) / plan.rows * ((N + columns - 1) / columns);
    }
    std::printf("%d %d %lld %lld\n", plan.rows, plan.splits, tiles, launches);
  }
}
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    d = tmp_path_factory.mktemp("launches")
    src, exe = str(d / "launches.cpp"), str(d / "launches")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2601_07396_amd", "csrc"), "-o", exe, src], check=True)

    def run(products):
        text = "\n".join(" ".join(str(int(x)) for x in p) for p in products)
        out = subprocess.run([exe], input=text, stdout=subprocess.PIPE, text=True, check=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    return run


def test_every_documented_size_has_a_way(launches):
    """M up to 2^31 - 1, N up to 2^24 (2^20 in 8 bits), K up to 2^20: some way, of launches that hold their tiles; and one launch wherever 2^22 tiles are enough."""
    rng = random.Random(2)
    top = (1 << 31) - 1
    products = [(M, N, K, dtype, act) for M in (1, 1 << 22, 536870912, 536870913, 1073741825, top) for N in (1, 3, 129, 1 << 20, 1 << 24) for K in (1, 128, 1 << 20)
                for dtype in range(3) for act in range(3) if dtype != E4M3 or N <= 1 << 20]
    products += [(int(2 ** rng.uniform(0, 31)), int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 20)), rng.randrange(3), rng.randrange(3)) for _ in range(50000)]
    for p, (rows, splits, tiles, n) in zip(products, launches(products)):
        assert rows in (16, 32, 64, 128, 256) and splits >= 1 and n >= 1, p
        assert 1 <= tiles <= 1 << 22, p
        wide = p[1] // (64 if p[3] == F32 or p[4] == 2 else 128) + 1
        assert n == 1 or (p[0] // 128 + 1) * wide * 2 > 1 << 22, p


@pytest.mark.gpu
@pytest.mark.parametrize("M,dtype,act", [((1 << 29) + 333, torch.float32, "none"), ((1 << 29) + 77, torch.float32, "swiglu"), ((1 << 30) + 333, torch.bfloat16, "none"),
                                         ((1 << 30) + 77, torch.bfloat16, "gelu")])
def test_rows_of_a_second_launch(M, dtype, act):
    """Zeros but for the rows around the end of a launch's 2^22 tiles: those as of a small product of the same rows, the others what the bias gives.

    Rows of A are normal and those of W of norm 1, so S = sum |a w| <= 14 and T^2 = sum (a w)^2 <= 4: float32 sums are 3 * 2^-21 * 14 = 2e-5 off on either side, and the gate's
    product of two of size 5 with slopes to 1.1 11 times that; those for bfloat16 7 * 2^-13 * sqrt(7 / 3) * 2 = 2.7e-3 on either side.  Results in bfloat16 may round to neighbours."""
    N, K, rows = 3, 128, 700
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < M * (K + 4 + 4 * N) + (16 << 30):
        pytest.skip("needs a device with more free memory")
    A = torch.zeros(M, K, device="cuda", dtype=torch.uint8)
    As = torch.full((M, 4), 127, device="cuda", dtype=torch.uint8)
    g = torch.Generator("cuda").manual_seed(M)
    q, s = svdc.quantize8(torch.randn(rows, K, device="cuda", generator=g))
    A[-rows:], As[-rows:] = q.view(torch.uint8), s.view(torch.uint8)
    W, Ws = svdc.quantize8(torch.randn(2 * N if act == "swiglu" else N, K, device="cuda", generator=g) / K ** 0.5, 128)
    bias = torch.randn(W.shape[0], device="cuda", generator=g)
    got = svdc.matmul8(A.view(torch.float8_e4m3fn), As.view(torch.float8_e8m0fnu), W, Ws, K, bias, dtype, act)
    want = svdc.matmul8(q, s, W, Ws, K, bias, dtype, act).double()
    empty = svdc.matmul8(*svdc.quantize8(torch.zeros(1, K, device="cuda")), W, Ws, K, bias, dtype, act).double()
    step, off = (2.0 ** -7, 6e-3) if dtype == torch.bfloat16 else (2.0 ** -17, 5e-4)
    assert ((got[-rows:].double() - want).abs() <= step * want.abs() + off).all()
    for i in range(0, M - rows, 1 << 26):
        part = got[i:min(i + (1 << 26), M - rows)].double()
        assert bool(((part - empty).abs() <= step * empty.abs()).all()), i
    del A, As, got, part
    torch.cuda.empty_cache()
