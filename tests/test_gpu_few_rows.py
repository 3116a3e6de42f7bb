"""bf16 linear layers of a few rows whose K is so short that waves of a workgroup have no turn of it, on the GPU
against the fp64 oracle, to the bounds of test_gpu_linear.py."""

import pytest
import torch

from paper_2507_16697_amd import ringx

from test_gpu_linear import check_backward, check_forward, make

pytestmark = pytest.mark.gpu


# Blocks of 16 rows and of 16 features that a workgroup takes: 1 x 1, 2 to 4 x 1, and past 4096 features 2 to 4 x 2.
# A wave's turn is 32 to 128 of K, four waves to a workgroup.
@pytest.mark.parametrize("O", [40, 4096, 4104, 8200])
@pytest.mark.parametrize("K", [8, 16, 32, 40, 64, 96, 128, 160])
@pytest.mark.parametrize("M", [1, 16, 17, 32, 33, 40, 48, 49, 50, 64])
def test_short_rows(M, K, O):
    x, w, b, res, _ = make(M + K + O, (M,), K, O, "bf16")
    y, pre = ringx.ringx_linear(x, w, b, act="gelu", residual=res, need_pre=True)
    check_forward(x, w, b, "gelu", res, "bf16", y, pre)
    for _ in range(10):
        again = ringx.ringx_linear(x, w, b, act="gelu", residual=res, need_pre=True)
        assert torch.equal(y, again[0]) and torch.equal(pre, again[1])


@pytest.mark.parametrize("lead,K,O,heads,pad", [((2, 25), 16, 64, 2, 0), ((2, 32), 64, 4104, 4, 0),
                                               ((3, 15), 32, 8200, 1, 0), ((60,), 24, 48, 0, 40),
                                               ((36,), 64, 8200, 0, 8)])
def test_short_rows_of_heads_and_of_wider_rows(lead, K, O, heads, pad):
    x, w, b, res, dy = make(K + O, lead, K, O, "bf16", heads, pad)
    y, pre = ringx.ringx_linear(x, w, b, act="silu", residual=res, need_pre=True)
    check_forward(x, w, b, "silu", res, "bf16", y, pre)
    check_backward(x, w, dy, pre, "silu", "bf16", *ringx.ringx_linear_bwd(x, w, dy, pre=pre, act="silu", bias=b))


def test_among_other_work():
    # products of many workgroups on another stream keep the memory busy meanwhile
    sets = [make(i, (M,), K, O, "bf16") for i, (M, K, O) in
            enumerate([(64, 8, 64), (50, 32, 40), (64, 64, 4104), (40, 32, 4104), (48, 64, 8200)])]
    ref = [ringx.ringx_linear(x, w, b)[0] for x, w, b, _, _ in sets]
    big = torch.randn(4096, 4096, device="cuda").to(torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(8):
            ringx.ringx_linear(big, big)
    got = [[ringx.ringx_linear(x, w, b)[0] for x, w, b, _, _ in sets] for _ in range(20)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for out in got for p, q in zip(ref, out))


# Both sides of the rule between the kernel for a few rows and the tiles: 16384 of K for every 16 rows, 2048 where
# the weights' rows are no whole pieces of 16 bytes, 1024 where only those of x are not.
@pytest.mark.parametrize("O", [40, 4104])
@pytest.mark.parametrize("M,K,pad", [
    (1, 16384, 0), (1, 16392, 0), (16, 16384, 0), (16, 16392, 0), (17, 8192, 0), (32, 8200, 0), (33, 5456, 0),
    (48, 5464, 0), (49, 4096, 0), (64, 4104, 0), (64, 8192, 8),
    (1, 2047, 0), (16, 2049, 0), (32, 1023, 0), (17, 1025, 0), (48, 682, 0), (33, 683, 0), (64, 511, 0), (49, 513, 0),
    (64, 4095, 0),
    (16, 1024, 3), (1, 1032, 3), (17, 512, 1), (32, 520, 1), (64, 256, 5), (49, 264, 5)])
def test_both_sides_of_the_rule(M, K, pad, O):
    x, w, b, res, _ = make(M + K + O, (M,), K, O, "bf16", pad=pad)
    y, pre = ringx.ringx_linear(x, w, b, act="gelu_tanh", residual=res, need_pre=True)
    check_forward(x, w, b, "gelu_tanh", res, "bf16", y, pre)
    assert torch.equal(y, ringx.ringx_linear(x, w, b, act="gelu_tanh", residual=res)[0])


@pytest.mark.parametrize("lead,K,O,heads", [
    ((1, 64), 8192, 72, 64), ((4, 4), 16448, 40, 257), ((2, 20), 6144, 4104, 96), ((1, 16), 1040, 40, 260),
    ((2, 8), 1020, 40, 255), ((3, 1), 32768, 24, 16)])
def test_both_sides_of_the_rule_of_heads(lead, K, O, heads):
    x, w, b, res, _ = make(K + O, lead, K, O, "bf16", heads)
    y, pre = ringx.ringx_linear(x, w, b, act="silu", residual=res, need_pre=True)
    check_forward(x, w, b, "silu", res, "bf16", y, pre)


def test_captured_on_the_other_side_of_the_rule():
    sets = [make(i, (M,), K, O, "bf16") for i, (M, K, O) in
            enumerate([(64, 8192, 264), (16, 32768, 40), (33, 2047, 136)])]

    def step():
        return [ringx.ringx_linear(x, w, b, residual=res)[0] for x, w, b, res, _ in sets]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(3):
        for i, (x, w, b, res, _) in enumerate(sets):
            x.copy_(make(10 * seed + i, (x.shape[0],), w.shape[1], w.shape[0], "bf16")[0])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, step()))
