"""Direct global -> LDS loads of the linear layer's kernels in the generated gfx950 code (CPU only: hipcc
cross-compiles).  They are inline assembly, for which the compiler inserts no waits."""

import os
import re
import shutil

import pytest

from test_build_isa import _asm

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                                reason="hipcc not available")


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    made = {}

    def get(src):
        if src not in made:
            made[src] = _asm(src, tmp_path_factory.mktemp("isa"))
        return made[src]
    return get


def kernels(text, fragment):
    """Names and lines (instructions and labels) of the kernels whose name has `fragment`."""
    found = re.findall(rf"^(_ZN\S*{fragment}\S*):(.*?)\.Lfunc_end", text, re.S | re.M)
    assert found, fragment
    lines = {name: [l.split(";")[0].strip() for l in body.splitlines()] for name, body in found}
    return {n: [l for l in ls if l and (l.startswith(".LBB") or not l.startswith("."))] for n, ls in lines.items()}


def reached_in_flight(lines):
    """Barriers and ends of the kernel that some path reaches from a direct load without a wait for all vector memory
    between the two, by line."""
    labels = {l[:-1]: i for i, l in enumerate(lines) if l.endswith(":")}
    seen, todo, bad = set(), [(0, False)], set()
    while todo:
        i, flying = todo.pop()
        if i >= len(lines) or (i, flying) in seen:
            continue
        seen.add((i, flying))
        op = lines[i].split()[0]
        if re.match(r"(global|buffer)_load\S*$", op) and re.search(r"_lds_| lds$", lines[i]):
            flying = True
        elif op == "s_waitcnt" and "vmcnt(0)" in lines[i]:
            flying = False
        elif flying and op in ("s_barrier", "s_endpgm"):
            bad.add(i)
        if op == "s_endpgm":
            continue
        if op.startswith(("s_branch", "s_cbranch")):
            todo.append((labels[lines[i].split()[1]], flying))
        if op != "s_branch":
            todo.append((i + 1, flying))
    return sorted(bad)


def test_the_search_itself():
    load, wait = "global_load_lds_dwordx4 v[0:1], off", "s_waitcnt vmcnt(0)"
    assert reached_in_flight([load, "s_barrier", "s_endpgm"]) == [1, 2]
    assert reached_in_flight([load, wait, "s_barrier", "s_endpgm"]) == []
    assert reached_in_flight([load, "s_cbranch_scc1 .LBB0_1", wait, ".LBB0_1:", "s_barrier", wait, "s_endpgm"]) == [4]
    assert reached_in_flight([load, "s_waitcnt vmcnt(3) lgkmcnt(0)", "s_barrier", wait, "s_endpgm"]) == [2]


def test_few_rows_has_no_load_in_flight_at_a_barrier(asm):
    """What the waves loaded into is what their sums are joined in, behind the first barrier: a load that is still in
    flight there, a wave's that has no turn of K included, would overwrite them."""
    some = kernels(asm("linear.hip"), "few_rows_kernel")
    with_loads = [n for n, ls in some.items() if any("_load_lds_" in l for l in ls)]
    assert len(with_loads) == 14     # seven forms of blocks, four waves and eight
    for name in with_loads:
        assert not reached_in_flight(some[name]), name


@pytest.mark.parametrize("src,load", [
    ("linear.hip", r"global_load_lds_dwordx4 v\[\d+:\d+\], off$"),
    ("gemm_bf16.hip", r"buffer_load_dwordx4 v\d+, s\[\d+:\d+\], 0 offen lds$"),
    ("gemm_f32.hip", r"buffer_load_dwordx4 v\d+, s\[\d+:\d+\], 0 offen lds$")])
def test_m0_only_feeds_direct_loads(src, load, asm):
    code = [l.split(";")[0].strip() for l in asm(src).splitlines()]
    code = [l for l in code if l and not l.startswith(".")]
    uses = [i for i, l in enumerate(code) if re.search(r"\bm0\b", l)]
    assert uses and len(uses) == sum(bool(re.match(load, l)) for l in code)
    for i in uses:
        assert re.match(r"s_mov_b32 m0, s\d+$", code[i]), code[i]
        assert code[i + 1] == "s_nop 0", code[i + 1]
        assert re.match(load, code[i + 2]), code[i + 2]


# (source, part of the kernel's name, kernels, products along r that each holds)
PRODUCTS = [("gemm_bf16.hip", "gemm_bf16_kernel", 9, 1), ("gemm_bf16.hip", "gemm_pair_kernel", 2, 2),
            ("gemm_f32.hip", r"gemm_f32_kernel\S*Li(?:128|64)E", 6, 1),
            ("gemm_f32.hip", r"gemm_f32_pair_kernel\S*Li64E", 1, 2)]


@pytest.mark.parametrize("src,fragment,count,products", PRODUCTS)
def test_a_step_waits_for_its_loads_once(src, fragment, count, products, asm):
    """The loop of a product of tiles, from its first matrix instruction to its last, waits for vector memory once,
    right before its barrier: a wait beside the products would be one for the loads of a later step."""
    some = kernels(asm(src), fragment)
    assert len(some) == count
    for name, lines in some.items():
        at = [i for i, l in enumerate(lines) if l.startswith("v_mfma")]
        # a kernel of two products has two loops, far apart
        cuts = [0] + [k for k in range(1, len(at)) if at[k] - at[k - 1] > 300] + [len(at)]
        loops = [lines[at[a]:at[b - 1]] for a, b in zip(cuts, cuts[1:])]
        assert len(loops) == products, name
        for loop in loops:
            waits = [i for i, l in enumerate(loop) if l.startswith("s_waitcnt") and "vmcnt" in l]
            assert len(waits) == 1 and "vmcnt(0)" in loop[waits[0]], name
            assert any(l == "s_barrier" for l in loop[waits[0]:waits[0] + 4]), name
