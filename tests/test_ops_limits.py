"""The largest calls of the layer operators beside the stage calls, where a launch would have 2^32 threads or more.  Nothing is launched here."""
import pytest

import __graft_entry__
from paper_2604_27085_amd import build as _build
import os
if not os.path.exists(_build.LIB):
    __graft_entry__.build()
from paper_2604_27085_amd import binding as B  # noqa: E402

P = 4096      # an address that is never followed: every call below is refused before anything is enqueued


def forward(batch, seq_q, seq_kv, d):
    B.rp_op_cross_attn_fwd(None, P, P, P, P, None, d, d, d, d, None, None, batch, seq_q, seq_kv, 1, 1, d, 0.1)


def backward(batch, seq_q, seq_kv, d):
    B.rp_op_cross_attn_bwd(None, P, P, P, P, P, P, P, P, P, P, d, d, d, d, d, d, d, d, None, None, batch, seq_q, seq_kv, 1, 1, d, 0.1)


@pytest.mark.parametrize("call,batch,seq_q,seq_kv,d", [
    (forward, 1 << 24, 1, 1, 64), (forward, 1 << 23, 129, 1, 64), (backward, 1 << 24, 1, 1, 64), (backward, 1 << 23, 1, 1, 128), (backward, 1 << 22, 1, 129, 128),
    (backward, 1 << 23, 1, 129, 64)])
def test_cross_attention_refuses_more_blocks_than_a_launch_has(call, batch, seq_q, seq_kv, d):
    with pytest.raises(B.RpError) as e:
        call(batch, seq_q, seq_kv, d)
    assert e.value.code == B.RP_EINVAL


def test_cross_attention_scratch_goes_as_far_as_the_forward():
    assert B.rp_op_cross_attn_scratch((1 << 24) - 1, 1, 1, 1, 1, 64) == (0, 0)
    with pytest.raises(B.RpError):
        B.rp_op_cross_attn_scratch(1 << 24, 1, 1, 1, 1, 64)


def test_balance_counts_tokens_up_to_two_to_the_30():
    """Token numbers, and the sums of one and a block's step, stay inside 31 bits."""
    args = [None, P, P, None, 1 << 30, 1, 16, 2, 0.1, 0.0, 1.0, P, P, P, None, P, P, 1 << 62]
    assert B.rp_op_moe_balance_scratch(1 << 30, 1 << 30, 16) > 0
    for T in ((1 << 30) + 1, 2 ** 31 - 1):
        args[4] = T
        assert B.lib.rp_op_moe_balance(*args) == B.RP_EINVAL
        with pytest.raises(B.RpError):
            B.rp_op_moe_balance_scratch(T, 1, 16)
