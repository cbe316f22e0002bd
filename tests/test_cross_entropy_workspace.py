"""The workspace of the cross entropy's forward pass has a bound that does not grow with rows times classes (no GPU needed)."""
import pytest

from paper_2401_06197_amd import binding as dcn

MOST = 1 << 20                                                # rows


@pytest.mark.parametrize("P", [1, 1000, 8192, 100_003, 1 << 18, MOST])
@pytest.mark.parametrize("V", [2, 150, 10_007, 40_009, 700_001, 1 << 22])
@pytest.mark.parametrize("K", [16, 1024])
def test_forward_workspace_is_bounded(P, V, K):
    # a maximum and a sum of 8 bytes for each of 2^25 (row, tile of classes), rounded up by 255 classes, of which a tile has 64 at
    # least; per row 8 bytes of what pieces have in common and 4 of the target's logit; 256 each of alignment
    row = min(8 * (1 << 25), 8 * P * (V // 64 + 1)) + 4 * 8 * P + 12 * P + 6 * 256
    assert dcn.dcnv4_linear_cross_entropy_workspace_bytes(P, K, V, dcn.DCNV4_F16, False) <= row
    # x and up to 2^27 numbers of w (255 classes more by rounding) in three bf16 parts, K in multiples of 32
    wide = (K + 31) // 32 * 32
    split = 6 * P * wide + 6 * min((1 << 27) + 255 * wide, V * wide) + 6 * 256
    assert dcn.dcnv4_linear_cross_entropy_workspace_bytes(P, K, V, dcn.DCNV4_F32, False) <= row + split
