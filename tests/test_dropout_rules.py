"""The host rules that cut the launches of the dropout and norm-rotation entry points (ringx_kernels.h),
compiled and asked on the CPU: no part of a sweep is empty, every choice is one of the forms that exist,
and the cuts measured to win are taken."""

import os
import random
import shutil
import subprocess

import pytest

from paper_2507_16697_amd import build as B

ROCM_INCLUDE = "/opt/rocm/include"
pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(ROCM_INCLUDE),
                                reason="needs g++ and the HIP headers")

MAIN = r"""
#include <cstdio>
#include "ringx_kernels.h"
int main() {
  using namespace ringx;
  long long bkv, bh, Nq, Nk, d;
  while (std::scanf("%lld %lld %lld %lld %lld", &bkv, &bh, &Nq, &Nk, &d) == 5) {
    const DropCut c = drop_cut(bkv, bh, Nq, Nk, d, true), s = drop_cut(bkv, bh, Nq, Nk, d, false);
    const RopeGrid f = rope_grid(bh * Nq, (int)(bh + 2 * bkv), 64 / rope_lanes(d, true), false);
    const RopeGrid b = rope_grid(bh * Nq, (int)(bh + 2 * bkv), 64 / rope_lanes(d, true), true);
    std::printf("%d %d %d %d %d %d %d %d %lld %lld %lld %lld\n", c.ks, c.kv, c.q, s.ks, s.kv, s.q,
                drop_fwd_streams(bh, Nq, Nk, d), drop_fwd_split(bh, Nq, Nk, d), (long long)f.x,
                (long long)f.y, (long long)b.x, (long long)b.y);
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("rules")
    (tmp / "m.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", ROCM_INCLUDE, "-I", B.CSRC,
                    "-I", B.INCLUDE, str(tmp / "m.cpp"), "-o", str(tmp / "m")], check=True)

    def run(shapes):
        text = "\n".join(" ".join(map(str, s)) for s in shapes)
        out = subprocess.run([str(tmp / "m")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return run


def test_no_part_is_empty_and_every_form_exists(ask):
    g = random.Random(5)
    size = lambda hi: int(round(hi ** g.random()))   # noqa: E731
    shapes = []
    for _ in range(4000):
        bkv = size(64)
        shapes.append((bkv, bkv * g.choice([1, 1, 2, 4, 8]), size(40000), size(300000), g.choice([64, 128])))
    shapes += [(1, 1, 1, 1, 64), (1, 64, 1, 40000, 128), (1, 1, 40000, 1, 64), (2048, 2048, 1, 1, 64),
               (1, 1, (1 << 31) - 128, 1 << 31, 64)]
    for (bkv, bh, Nq, Nk, d), r in zip(shapes, ask(shapes)):
        ks, kv, q, sks, skv, sq, fks, fq, fx, fy, bx, by = r
        assert ks in (1, 2, 4) and sks in (1, 2, 4) and fks in (1, 2, 4)
        assert skv == sq == 1
        # a part holds a tile of 128 queries, or of 512 keys; parts of dQ go with four streams
        assert 1 <= kv <= max(1, Nq // 128) and 1 <= q <= max(1, Nk // 512) and (q == 1 or ks == 4)
        assert 1 <= fq <= max(1, Nk // 512) and max(kv, q, fq) <= 32
        # a stream holds a tile
        assert all(s == 1 or Nk >= 64 * s for s in (ks, sks, fks))
        # every token has a workgroup, every share of heads a head
        per = 4 * 64 // (d // 8)
        assert fx == -(-bh * Nq // per) and bx == min(fx, 2048)
        assert 1 <= fy <= bh + 2 * bkv and 1 <= by <= bh + 2 * bkv


@pytest.mark.parametrize("shape,cut", [
    ((16, 16, 4096, 32768, 128), (1, 1, 1)), ((16, 16, 16384, 16384, 64), (1, 1, 1)),
    ((16, 16, 4096, 4096, 64), (1, 1, 1)), ((8, 8, 4096, 4096, 128), (2, 1, 1)),
    ((2, 2, 4096, 4096, 128), (4, 2, 1)), ((1, 8, 2048, 8192, 128), (2, 2, 1)),
    ((1, 4, 1000, 30000, 64), (4, 1, 4)), ((2, 2, 200, 700, 128), (4, 1, 1))])
def test_measured_cuts(ask, shape, cut):
    """(dQ streams, parts of dK/dV, parts of dQ)"""
    assert ask([shape])[0][:3] == cut
