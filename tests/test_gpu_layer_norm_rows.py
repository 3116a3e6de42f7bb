"""What the layer norm keeps of rows that hold infinities or NaN, on the GPU."""

import pytest
import torch

from paper_2507_16697_amd import ringx

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.mark.parametrize("store", ["bf16", "fp32"])
@pytest.mark.parametrize("C", [1, 7, 64, 300, 1024, 2047, 8192, 16384])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_statistics_of_rows_that_are_not_finite(value, C, store):
    g = torch.Generator(device="cuda").manual_seed(C)
    x = torch.randn(7, C, generator=g, device="cuda").to(DT[store])
    ref, kept = ringx.ringx_layer_norm(x)
    bad = x.clone()
    bad[1, C - 1] = bad[4, 0] = value
    y, stats = ringx.ringx_layer_norm(bad)
    rows = torch.zeros(7, dtype=torch.bool, device="cuda")
    rows[1] = rows[4] = True
    # neither a mean nor a deviation
    assert torch.isnan(stats[:, rows]).all()
    assert torch.isnan(y[rows]).all()
    # the others are as they were
    assert torch.equal(stats[:, ~rows], kept[:, ~rows]) and torch.equal(y[~rows], ref[~rows])
    # and the gradients say so: of these rows, and of all weights
    w, b = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    dy = torch.randn(7, C, generator=g, device="cuda").to(DT[store])
    dx, dw, db = ringx.ringx_layer_norm_bwd(bad, dy, stats, w, b)
    assert torch.isnan(dx[rows]).all() and torch.isfinite(dx[~rows]).all()
    assert torch.isnan(dw).all() and torch.isfinite(db).all()


def test_the_widest_rows_are_summed_as_a_tree():
    # 1024 threads of 16 values: 15 additions in a thread, 6 over its wave's lanes, 4 over 16 waves; each rounds by at
    # most E = 2^-24 of the sum.  g = 1 in the first thread's first column and 2^-24 wherever an addition to 1 would
    # lose it: the thread's other columns (pieces of 4, 4096 apart), lanes 1, 2, 4, 8, 16 and 32, and every other wave
    # (with the waves one after the other the loss would be 36 E).
    C, E = 16384, 2.0 ** -24
    at = [4096 * v + j for v in range(4) for j in range(4)][1:]
    at += [4 * lane for lane in (1, 2, 4, 8, 16, 32)] + [4 * 64 * wave for wave in range(1, 16)]
    dy = torch.zeros(3, C, device="cuda")
    dy[:, 0] = 1.0
    dy[:, at] = E
    zero = 4096 + 5       # a column with g = 0
    assert dy[0, zero] == 0 and len(set(at)) == 36
    x, stats = torch.zeros(3, C, device="cuda"), torch.zeros(2, 3, device="cuda")
    stats[1] = 1.0        # n = 0: dx = g - sum g / C, and C is a power of two
    dx, _, _ = ringx.ringx_layer_norm_bwd(x, dy, stats)
    got = -dx[:, zero].double() * C
    assert ((got - (1 + 36 * E)).abs() <= 25 * E * (1 + 36 * E)).all(), ((got - 1) / E).tolist()
