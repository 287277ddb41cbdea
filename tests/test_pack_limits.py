"""Sizes at the edges of what the operators for training on packed documents take.  Nothing is launched here."""
import pytest

from test_pack_refusals import B, Bytes, P, refused


@pytest.mark.parametrize("T", [129, 8192, 8193, 9000, 9217, 70000, 300000])
@pytest.mark.parametrize("V", [1, 2, 3, 5, 1000, 1 << 19])
@pytest.mark.parametrize("h", [8, 24])
def test_the_parts_of_the_embedding_scratch_are_on_16_byte_boundaries(T, V, h):
    """Every part but the last is rounded up to 16 bytes, and the last is fp32 rows of a multiple of 8: so is the sum.  (One or two digits of few values, counted by an odd number of blocks: 72 bytes.)"""
    assert B.rp_op_embed_scratch(T, V, h) % 16 == 0


def test_dropout_refuses_more_blocks_than_a_launch_has():
    """131073 x 1048568 elements, 8 (2^34 - 1) of them: 2^24 blocks of 256 threads."""
    refused(B.rp_op_dropout, x=P, ldx=1048568, res=None, ldr=1048568, y=2 * P, ldy=1048568, T_=131073, n=1048568, p=0.1, seed=1, stream=None)
