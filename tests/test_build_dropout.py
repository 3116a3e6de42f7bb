"""Properties of the generated gfx950 code of the kernels with dropout and of the norm with rotation
(CPU only: hipcc cross-compiles): the same rules as for the kernels without."""

import os
import re
import shutil

import pytest

from test_build_isa import _asm, _resources, test_m0_only_feeds_direct_lds_loads as _m0_rule

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                                reason="hipcc not available")

DROP_BF16 = ["fwd_drop_bf16.hip", "bwd_drop_bf16.hip"]
# (part of the kernel's name, workgroups that share a CU, waves of one); every kernel matching keeps its
# values in registers.  A wave of w per SIMD has 512 / w registers, in steps of 8; a CU has 160 KiB of LDS.
NO_SCRATCH = {
    "fwd_drop_bf16.hip": [(r"fwd_bf16_drop_kernelILi64E", 1, 8)],
    "bwd_drop_bf16.hip": [(r"bwd_drop_kernelILi64E", 1, 8)],
    "fwd_drop_f32.hip": [(r"fwd_f32_drop_kernel", 1, 4)],
    "bwd_drop_f32.hip": [(r"bwd_f32_drop_kernelILi[1-5]E", 2, 4)],
    # the backward's measured splits count on 4 waves on a SIMD
    "norm_rope.hip": [(r"norm_rope_kernel", 4, 4), (r"norm_rope_bwd_kernel", 4, 4),
                      (r"weight_grad_kernel", 4, 4)],
}


@pytest.mark.parametrize("src", DROP_BF16)
def test_m0_only_feeds_direct_lds_loads(src, tmp_path):
    _m0_rule(src, tmp_path)


@pytest.mark.parametrize("src", sorted(NO_SCRATCH))
def test_instructions_and_registers(src, tmp_path):
    text = _asm(src, tmp_path)
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text)
    assert not re.search(r"^\s*flat_(load|store|atomic)", text, re.M)
    res = _resources(text)
    for frag, groups, waves in NO_SCRATCH[src]:
        names = [n for n in res if re.search(frag, n)]
        assert names, frag
        for n in names:
            vgpr, scratch, lds = res[n]
            per_simd = max(1, groups * waves // 4)
            assert scratch == 0, (n, scratch)
            assert vgpr <= 512 // per_simd // 8 * 8 and groups * lds <= 160 * 1024, (n, vgpr, lds)
