"""Limits of the dropout entry points, on the host (pointers are never dereferenced)."""

import numpy as np
import pytest

from paper_2507_16697_amd import ringx

from test_dropout_host import BF16, DROPOUT, SHAPE, WORKSPACE, bstep, bwd, fstep, fwd, needs_lib

LAUNCH = 1 << 23      # workgroups of 512 threads: a launch has fewer than 2^32 threads


@needs_lib
@pytest.mark.parametrize("d", [64, 128])
def test_backward_is_refused_where_one_launch_cannot_take_it(d):
    """dK/dV's workgroups (128 keys of a K/V head) and dQ's (256 queries of a head) share a launch.  What fits
    goes on to the next check, here that of the workspace."""
    size = ringx.ringx_bwd_drop_workspace_bytes
    half = LAUNCH // 2
    for n, Hkv, H, Nq, Nk in ((LAUNCH, half, half, 1, 1), (LAUNCH - 2, half - 1, half - 1, 1, 1),
                              (LAUNCH, 1, LAUNCH - 1, 1, 1), (LAUNCH - 1, 1, LAUNCH - 2, 1, 1),
                              (LAUNCH, 4, half - 4, 257, 256)):
        assert Hkv * ((Nk + 127) // 128) + H * ((Nq + 255) // 256) == n
        got = bwd(B=1, H=H, Hkv=Hkv, Nq=Nq, Nk=Nk, d=d, wsb=16)
        assert got == (SHAPE if n >= LAUNCH else WORKSPACE), (n, Hkv, H)
        assert (size(1, H, Hkv, Nq, Nk, d, BF16) == 0) == (n >= LAUNCH)
    assert bstep(B=2, H=LAUNCH // 4, Nq=1, Nk=1, d=d) == SHAPE
    # far beyond: no time is spent on how such a launch would be cut
    assert bwd(B=1, H=1 << 30, Hkv=1 << 30, Nq=1, Nk=1, d=d, wsb=16) == SHAPE


@needs_lib
def test_rates_at_the_ends_of_the_range():
    """256 p rounds to nearest, ties to even: 1/512 rounds to no rate and 511/512 to all; the status text names
    the range as it is.  What is accepted goes on to the next check, here that of the workspace."""
    lo, hi = np.float32(1 / 512), np.float32(511 / 512)
    up, down = np.nextafter(lo, np.float32(1)), np.nextafter(hi, np.float32(0))
    for p in (lo, np.nextafter(lo, np.float32(0)), hi, np.nextafter(hi, np.float32(1))):
        for fn in (fwd, fstep, bwd, bstep):
            assert fn(p=float(p)) == DROPOUT, p
    for p in (0.0, up, down, 1 / 256, 255 / 256):
        assert bwd(p=float(p), wsb=16) == WORKSPACE, p
    text = ringx.ringx_status_str(DROPOUT)
    assert "excluded" in text and "1/512" in text and "511/512" in text and "[" not in text
