"""Which dropout kernels keep values in memory (scratch) and how many bytes a lane (CPU only: hipcc
cross-compiles).  The rules of test_build_dropout.py cover the forms without any.  These hold more than the
256 registers of a wave (two waves on a SIMD):

  * bf16, d = 128: the generator's state and the masks come on top of kernels that fill the registers by
    themselves (the four-stream step form has its 88 bytes without dropout too).  All of it is written and
    read outside the tile loops, once a launch.
  * fp32 backward, d > 80: four fragments, two accumulators and the generator.  Without dropout it is 16 to
    196 bytes from d = 97 on, for the same reason; fewer rows a wave would read the other side more often."""

import os
import re
import shutil

import pytest

from test_build_isa import _asm, _resources

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                                reason="hipcc not available")

# part of the kernel's name, most bytes a lane
SCRATCH = {
    "fwd_drop_bf16.hip": [(r"ILi128ELi0ELi1E", 8), (r"ILi128ELi0ELi[24]E", 0), (r"ILi128ELi2ELi[12]E", 0),
                          (r"ILi128ELi2ELi4E", 88)],
    "bwd_drop_bf16.hip": [(r"ILi128ELi1E", 20), (r"ILi128ELi2E", 0), (r"ILi128ELi4E", 36)],
    "bwd_drop_f32.hip": [(r"ILi6E", 28), (r"ILi7E", 60), (r"ILi8E", 236)],
}


def _tile_loops(code):
    """Spans of the innermost loops that hold matrix products."""
    label = {l[:-1]: i for i, l in enumerate(code) if re.fullmatch(r"\.LBB\w+:", l)}
    spans = []
    for i, l in enumerate(code):
        to = re.match(r"s_c?branch\w*\s+(\.LBB\w+)", l)
        if to and label.get(to.group(1), i) < i:
            a = label[to.group(1)]
            if any(x.startswith("v_mfma") for x in code[a:i]):
                spans.append((a, i))
    return [s for s in spans if not any(t != s and s[0] <= t[0] and t[1] <= s[1] for t in spans)]


@pytest.mark.parametrize("src", sorted(SCRATCH))
def test_scratch(src, tmp_path):
    text = _asm(src, tmp_path)
    res = _resources(text)
    for frag, most in SCRATCH[src]:
        names = [n for n in res if re.search("drop_kernel" + frag, n)]
        assert names, frag
        for n in names:
            assert res[n][1] <= most and res[n][0] <= 256, (n, res[n])
            if "f32" in src:
                continue
            body = text[text.index("\n" + n + ":"):]
            code = [l.split(";")[0].strip() for l in body[:body.index("\n.Lfunc_end")].splitlines()]
            code = [l for l in code if l]
            loops = _tile_loops(code)
            assert loops, n
            spilled = [i for i, l in enumerate(code) if l.startswith("scratch_")]
            assert not any(a <= i <= b for i in spilled for a, b in loops), n
