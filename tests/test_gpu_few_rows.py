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


@pytest.mark.parametrize("lead,K,O,heads,pad", [((2, 25), 16, 64, 2, 0), ((2, 32), 64, 4104, 4, 0), ((3, 15), 32, 8200, 1, 0),
                                               ((60,), 24, 48, 0, 40), ((36,), 64, 8200, 0, 8)])
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
