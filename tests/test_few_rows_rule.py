"""Which bf16 linear layers of up to 64 rows take the kernel for a few rows and which the tiles (CPU only: by the
workspace that the tiles ask for, parts of a long r and copies of operands; the kernel for a few rows asks for none)."""

import pytest

from paper_2507_16697_amd import ringx

BF16 = ringx.RINGX_BF16


def tiles(M, K, O, ldx=None, heads=0, tokens=0):
    return ringx.ringx_linear_workspace_bytes(ldx or K, heads, tokens, M, K, O, BF16) > 0


# us of the kernel for a few rows and of the tiles, weights from HBM
@pytest.mark.parametrize("M,K,O,few,whole", [
    (64, 4096, 2048, 12.5, 16.9), (17, 8192, 2048, 17.8, 20.6), (32, 8192, 8192, 39.2, 44.1),
    (1, 16384, 1024, 17.3, 23.4), (16, 16384, 4096, 35.3, 40.3), (33, 4096, 8192, 21.7, 29.3),
    (64, 375, 2048, 11.2, 12.6), (17, 1023, 1024, 12.7, 16.1), (16, 2047, 2048, 19.7, 24.8), (1, 1, 1, None, None),
    (64, 8, 8, None, None)])
def test_a_few_rows(M, K, O, few, whole):
    assert few is None or few < whole
    assert not tiles(M, K, O)


@pytest.mark.parametrize("M,K,O,few,whole", [
    (64, 8192, 2048, 32.7, 20.7), (64, 8192, 1024, 19.4, 18.2), (17, 16384, 1024, 30.7, 23.4),
    (64, 6144, 2048, 26.8, 20.0), (16, 32768, 2048, 53.5, 42.1), (1, 65536, 64, 33.5, 26.2),
    (64, 65536, 512, 235.6, 35.7), (1, 2 ** 20, 16, 1229.8, 259.3), (64, 1023, 8192, 53.0, 27.5),
    (32, 2047, 8192, 60.1, 41.3), (2, 4095, 1024, 26.8, 25.6), (16, 8191, 2048, 73.4, 42.2),
    (64, 16383, 1024, 360.7, 45.7)])
def test_much_of_k(M, K, O, few, whole):
    assert whole < few
    assert tiles(M, K, O)


@pytest.mark.parametrize("M,K,O,few,whole", [(16, 2048, 8192, 41.1, 23.8), (64, 1024, 8192, 47.8, 16.1)])
def test_rows_that_come_in_no_whole_pieces(M, K, O, few, whole):
    assert whole < few
    assert tiles(M, K, O, ldx=K + 1) and not tiles(M, K, O, ldx=K + 8)
    assert not tiles(M, 64, O, ldx=65)
    # an attention's layout whose heads are no whole pieces
    assert tiles(M, K, O, heads=K // 4, tokens=M) and not tiles(M, K, O, heads=K // 64, tokens=M)
