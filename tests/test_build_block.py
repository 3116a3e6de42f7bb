"""Properties of the generated gfx950 code of the layer norm and of the linear layer's kernels (CPU only: hipcc
cross-compiles): the same rules as for the other kernels."""

import os
import re
import shutil

import pytest

from test_build_isa import _asm, _resources

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                                reason="hipcc not available")

# (part of the kernel's name, workgroups that share a CU, waves of one)
KERNELS = {
    # two waves on a SIMD; the backward of the widest rows, past 8192, is known to spill
    "layer_norm.hip": [(r"layer_norm_kernel", 1, 8), (r"layer_norm_bwd_kernel(?!.*ELi1024EEE)", 1, 8)],
    "linear.hip": [(r"few_rows_kernel", 1, 8), (r"grad_pass_kernel", 2, 4), (r"pack_kernel", 2, 4),
                   (r"join_kernel", 2, 4), (r"column_sums_kernel", 1, 16)],
    # two small workgroups, a large one, or one of two groups of waves
    "gemm_bf16.hip": [(r"gemm_bf16_kernel.*TileILi128ELi128ELi2ELi2ELi1E", 2, 4),
                      (r"gemm_bf16_kernel.*TileILi128ELi128ELi2ELi2ELi2E", 1, 8),
                      (r"gemm_bf16_kernel.*TileILi256E", 1, 8), (r"gemm_pair_kernel", 1, 8),
                      (r"gemm_join", 2, 4)],
    "gemm_f32.hip": [(r"gemm_f32_kernel.*ELi128E", 2, 4), (r"gemm_f32_(kernel|pair_kernel).*Li(64|32)E", 4, 4)],
}


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    made = {}

    def get(src):
        if src not in made:
            made[src] = _asm(src, tmp_path_factory.mktemp("isa"))
        return made[src]
    return get


@pytest.mark.parametrize("src", sorted(KERNELS))
def test_instructions_and_registers(src, asm):
    text = asm(src)
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text)
    assert not re.search(r"^\s*flat_(load|store|atomic)", text, re.M)
    assert not re.search(r"\b(global|flat|buffer)_atomic", text)     # sums have one order
    res = _resources(text)
    for frag, groups, waves in KERNELS[src]:
        names = [n for n in res if re.search(frag, n)]
        assert names, frag
        for n in names:
            vgpr, scratch, lds = res[n]
            per_simd = max(1, groups * waves // 4)
            assert scratch == 0, (n, scratch)
            assert vgpr <= 512 // per_simd // 8 * 8 and groups * lds <= 160 * 1024, (n, vgpr, lds)


def test_m0_only_feeds_direct_lds_loads(asm):
    code = [l.strip() for l in asm("gemm_bf16.hip").splitlines()]
    code = [l for l in code if l and not l.startswith((";", "."))]
    uses = [i for i, l in enumerate(code) if re.search(r"\bm0\b", l)]
    assert uses, "expected direct LDS loads"
    for i in uses:
        assert re.match(r"s_mov_b32 m0, s\d+$", code[i]), code[i]
        assert code[i + 1] == "s_nop 0", code[i + 1]
        assert re.match(r"buffer_load_dwordx4 v\d+, s\[\d+:\d+\], 0 offen lds$", code[i + 2]), code[i + 2]


def test_products_wait_for_their_operands_alone(asm):
    """Between two barriers of a product's loop the vector memory counter is waited for once: a wait beside
    the products would be one for the loads of a later step."""
    for name, body in re.findall(r"^(_ZN\S*gemm_bf16_kernel\S+):(.*?)\.Lfunc_end", asm("gemm_bf16.hip"), re.S | re.M):
        lines = [l.strip() for l in body.splitlines()]
        at = [i for i, l in enumerate(lines) if l.startswith("v_mfma")]
        loop = lines[at[0]:at[-1]]
        waits = [l for l in loop if l.startswith("s_waitcnt") and "vmcnt" in l]
        assert len(waits) == 1, (name, waits)
