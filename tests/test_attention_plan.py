"""How an attention is cut up (host arithmetic, compiled on its own: no GPU), and what the compiler gave the kernels."""
import os
import random
import subprocess

import pytest

import paper_2601_07396_amd as pkg
from test_kernel_resources import _kernels

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include "attention_plan.h"
// batch q_rows k_rows heads share head_dim dtype cus -> q_tiles units whole parts tiles_of_part, keys of a tile
int main() {
  long long batch, q, k;
  int heads, share, d, dtype, cus;
  while (std::scanf("%lld %lld %lld %d %d %d %d %d", &batch, &q, &k, &heads, &share, &d, &dtype, &cus) == 8) {
    svdc_attention p{};
    p.batch = batch, p.q_rows = q, p.k_rows = k, p.heads = heads * share, p.kv_heads = heads, p.head_dim = d, p.dtype = dtype;
    const svdc::AttentionPlan plan = svdc::attention_plan(p, cus);
    std::printf("%d %d %d %d %d %d\n", plan.q_tiles, plan.units, plan.whole, plan.parts, plan.tiles_of_part, svdc::attention_tile_keys(svdc::attention_width(d), dtype == 0));
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("plans")
    src, exe = str(d / "plan.cpp"), str(d / "plan")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2601_07396_amd", "csrc"), "-o", exe, src], check=True)

    def run(cases):
        text = "\n".join(" ".join(str(int(x)) for x in c) for c in cases)
        out = subprocess.run([exe], input=text, stdout=subprocess.PIPE, text=True, check=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    return run


def test_every_key_once(plans):
    """Units cover the queries, parts the keys, none of them is empty, and a lane each is enough to join them."""
    rng = random.Random(1)
    cases = [(1, 1, 1, 1, 1, 1, 0, 256), (1, 1, 0, 1, 1, 1, 1, 256), (1, 2 ** 30, 2 ** 30, 1, 1, 256, 0, 256), (1, 2 ** 14, 2 ** 30, 1, 2 ** 16, 256, 0, 256),
             (65535, 1, 2 ** 15, 128, 1, 64, 1, 256), (1, 1, 2 ** 30, 1, 1, 8, 1, 304)]
    for _ in range(4000):
        batch, heads = rng.choice([1, 1, 2, 5, 31]), rng.choice([1, 3, 8, 24, 40])
        cases.append((batch, int(2 ** rng.uniform(0, 17)), int(2 ** rng.uniform(0, 18)), heads, rng.choice([1, 1, 3, 8]), rng.choice([8, 64, 72, 128, 200, 256]), rng.randint(0, 1), rng.choice([1, 32, 256, 304])))
    for case, (q_tiles, units, whole, parts, each, keys) in zip(cases, plans(cases)):
        batch, q, k, heads, share, _, _, cus = case
        tiles = max(1, -(-k // keys))
        assert q_tiles == -(-q * share // 128) and units == batch * heads * q_tiles
        assert 0 <= whole <= units and 1 <= parts <= 64
        assert parts * each >= tiles and (parts - 1) * each < tiles, case
        assert (whole == units) == (parts == 1)
        assert units - whole < max(cus, 1), "a second launch for more than a round"
        assert whole + (units - whole) * parts < 2 ** 31


def test_few_rows_fill_the_card(plans):
    for case in ((1, 64, 119056, 24, 1, 128, 1, 256), (1, 1, 20000, 8, 1, 128, 1, 256), (1, 1, 20000, 8, 4, 128, 1, 256), (2, 100, 30000, 5, 1, 64, 0, 256)):
        (_, units, whole, parts, _, _), = plans([case])
        assert whole == 0 and units * parts > 256
    for case in ((1, 1, 60, 24, 1, 128, 1, 256), (1, 32768, 4096, 2, 1, 128, 1, 256), (1, 4096, 4096, 2, 8, 128, 1, 256)):      # one tile; two rounds exactly
        (_, units, whole, _, _, _), = plans([case])
        assert whole == units


@pytest.mark.parametrize("kernel,least", [("attention_kernelI", 32), ("attention_join_kernel", 8), ("norm_rotate_kernel", 60), ("rotary_table_kernel", 2)])
def test_no_scratch(kernel, least):
    """Sums, products and operands stay in registers; but for heads of more than 128 columns in float32 or at odd strides, which have more of them than there are registers."""
    if not os.path.exists(pkg.lib_path()):
        pytest.skip("the library is not built")
    found = {n: k[".private_segment_fixed_size"] for n, k in _kernels(pkg.lib_path()).items() if kernel in n}
    assert len(found) >= least
    assert {n: size for n, size in found.items() if size and not ("fLi256E" in n or "DF16bLi256ELb0E" in n)} == {}
