"""The layer norm and the linear layer at the most rows that they take, on the GPU: all rows but the first and last
ones are zero, which adds nothing to any sum."""

import pytest
import torch

from paper_2507_16697_amd import ringx

from test_gpu_linear import check_backward, check_forward, ends

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def sparse(M, C, g):
    t = torch.zeros(M, C, dtype=torch.bfloat16, device="cuda")
    at = ends(M)
    t[at] = torch.randn(len(at), C, generator=g, device="cuda").to(torch.bfloat16)
    return t


def test_linear_of_the_most_rows():
    M, K, O = 2 ** 31 - 1024, 8, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = sparse(M, K, g), sparse(M, O, g)
    w, b = torch.randn(O, K, generator=g, device="cuda").to(torch.bfloat16), torch.randn(O, generator=g, device="cuda")
    at = ends(M)
    y, _ = ringx.ringx_linear(x, w, b)
    check_forward(x[at], w, b, "none", None, "bf16", y[at], None)
    for i in range(64, M - 200, 2 ** 28):
        assert (y[i:min(i + 2 ** 28, M - 200)] == b.to(torch.bfloat16)).all()
    del y
    dx, dw, db = ringx.ringx_linear_bwd(x, w, dy, bias=b)
    check_backward(x[at], w, dy[at], None, "none", "bf16", dx[at], dw, db)
    for i in range(64, M - 200, 2 ** 28):
        assert not dx[i:min(i + 2 ** 28, M - 200)].any()


def test_layer_norm_of_more_rows_than_32_bits():
    M, C = 2 ** 31 + 300, 8
    g = torch.Generator(device="cuda").manual_seed(2)
    x = sparse(M, C, g)
    at = ends(M)
    w, b = (torch.randn(C, generator=g, device="cuda") for _ in range(2))
    y, stats = ringx.ringx_layer_norm(x, w, b)
    few, kept = ringx.ringx_layer_norm(x[at], w, b)
    assert torch.equal(y[at], few) and torch.equal(stats[:, at], kept)
    for i in range(64, M - 200, 2 ** 28):
        assert (y[i:min(i + 2 ** 28, M - 200)] == b.to(torch.bfloat16)).all()
    del y
    dy = sparse(M, C, g)
    dx, dw, db = ringx.ringx_layer_norm_bwd(x, dy, stats, w, b)
    gx, gw, gb = ringx.ringx_layer_norm_bwd(x[at], dy[at], kept, w, b)
    assert torch.equal(dx[at], gx)
    # sums of 264 terms in two orders, each off by at most 264 steps of 2^-24 of the terms' sizes; |n| is below 3
    size = dy[at].float().abs().sum(0)
    assert ((db - gb).abs() <= 2 * 264 * 2.0 ** -24 * size).all()
    assert ((dw - gw).abs() <= 2 * 264 * 2.0 ** -24 * 3 * size).all()
    for i in range(64, M - 200, 2 ** 28):
        assert not dx[i:min(i + 2 ** 28, M - 200)].any()
