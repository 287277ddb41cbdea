"""What the layer operators beside the stage calls refuse, and their 64-bit references against differences.  Nothing is launched here."""
import ctypes as C
import math

import pytest

import __graft_entry__
from paper_2604_27085_amd import build as _build
import os
if not os.path.exists(_build.LIB):
    __graft_entry__.build()
from paper_2604_27085_amd import binding as B  # noqa: E402

import ops_reference as R  # noqa: E402

torch = pytest.importorskip("torch")
P = 4096      # an address that is never followed: every call below is refused before anything is enqueued


def refused(f, *args, code=B.RP_EINVAL, **kw):
    with pytest.raises(B.RpError) as e:
        f(*args, **kw)
    assert e.value.code == code


def scaling(**kw):
    return B.make_rope_scaling(**kw)


@pytest.mark.parametrize("bad", [dict(kind=4), dict(kind=-1), dict(base=0.0), dict(base=math.inf), dict(base=math.nan), dict(kind=1, factor=0.0),
                                 dict(kind=2, factor=-1.0), dict(kind=3, slow=4.0, fast=4.0), dict(kind=3, trained_len=0), dict(kind=3, fast=math.inf),
                                 dict(amplitude=math.nan)])
def test_table_refuses_scalings(bad):
    refused(B.rp_op_rope_table_scaled, None, P, scaling(**bad), 8, 64)


def test_table_refuses_arguments():
    refused(B.rp_op_rope_table_scaled, None, None, scaling(), 8, 64)
    refused(B.rp_op_rope_table_scaled, None, P, scaling(), -1, 64)
    refused(B.rp_op_rope_table_scaled, None, P + 4, scaling(), 8, 64)
    for rot in (0, 1, 63, 514):
        refused(B.rp_op_rope_table_scaled, None, P, scaling(), 8, rot)
    refused(B.rp_op_rope_table_scaled, None, P, scaling(kind=2, factor=2.0), 8, 2)
    s = scaling()
    s.struct_size = 8
    refused(B.rp_op_rope_table_scaled, None, P, s, 8, 64)
    assert B.lib.rp_op_rope_table_scaled(None, P, None, 8, 64) == B.RP_EINVAL


GOOD_ROPE = dict(bwd=0, layout=0, d=64, rot=64, in_q=P, in_k=P, ld_in_q=256, ld_in_k=128, out_q=P, out_k=P, ld_out_q=256, ld_out_k=128, cs=P, n_pos=8,
                 pos=None, T_=8, seq=8, a=4, k=2)


@pytest.mark.parametrize("bad", [dict(layout=2), dict(layout=-1), dict(d=60), dict(d=0), dict(d=520, rot=64), dict(rot=0), dict(rot=63), dict(rot=66), dict(in_q=None),
                                 dict(in_k=None), dict(out_q=None), dict(out_k=P + 8), dict(in_q=P + 2), dict(ld_in_q=252), dict(ld_in_q=248), dict(ld_out_k=120),
                                 dict(ld_out_q=1 << 24), dict(cs=None), dict(cs=P + 4), dict(n_pos=7), dict(n_pos=-1), dict(T_=-1), dict(T_=(1 << 30) + 1, pos=P), dict(seq=0), dict(a=-1), dict(k=-1),
                                 dict(ld_out_q=264)])
def test_rope_refuses(bad):
    refused(B.rp_op_rope, None, **dict(GOOD_ROPE, **bad))


GOOD_CROSS = dict(q=P, k=P, v=P, o=P, lse=P, ldq=512, ldk=256, ldv=256, ldo=512, q_len=None, kv_len=None, batch=2, seq_q=3, seq_kv=5, a=4, kh=2, d=128, scale=0.1)
BAD_CROSS = [dict(q=None), dict(k=None), dict(v=None), dict(q=P + 8), dict(k=P + 2), dict(ldq=508), dict(ldq=504), dict(ldk=248), dict(ldv=1 << 24), dict(ldk=0),
             dict(batch=-1), dict(seq_q=-1), dict(seq_kv=-1), dict(a=0), dict(kh=0), dict(kh=3), dict(d=96), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan),
             dict(scale=math.inf), dict(seq_q=1 << 30), dict(seq_kv=1 << 30), dict(batch=1 << 30)]


@pytest.mark.parametrize("bad", BAD_CROSS + [dict(o=None), dict(o=P + 4), dict(ldo=0)])
def test_cross_forward_refuses(bad):
    refused(B.rp_op_cross_attn_fwd, None, **dict(GOOD_CROSS, **bad))


@pytest.mark.parametrize("bad", BAD_CROSS + [dict(dout=None), dict(lse=None), dict(delta=None), dict(dq=None), dict(dk=None), dict(dv=P + 8), dict(lddq=256),
                                             dict(lddo=500), dict(lddk=248), dict(lddv=1 << 24), dict(ldo=8)])
def test_cross_backward_refuses(bad):
    good = dict(GOOD_CROSS, dout=P, delta=P, dq=P, dk=P, dv=P, lddo=512, lddq=512, lddk=256, lddv=256)
    refused(B.rp_op_cross_attn_bwd, None, **dict(good, **bad))


def test_cross_scratch():
    with pytest.raises(B.RpError):
        B.rp_op_cross_attn_scratch(1, 1, 1, 3, 2, 64)
    assert B.rp_op_cross_attn_scratch(0, 0, 0, 4, 2, 64) == (0, 0)
    assert B.rp_op_cross_attn_scratch(1, 1, 0, 4, 2, 64) == (0, 0)
    assert B.rp_op_cross_attn_scratch(64, 4096, 4096, 32, 32, 128)[0] == 0      # rows enough for the chip
    f, b = B.rp_op_cross_attn_scratch(1, 1, 32768, 8, 8, 128)
    assert 0 < f <= b
    assert B.lib.rp_op_cross_attn_scratch(1, 1, 32768, 8, 8, 128, None, None) == B.RP_OK
    # a scratch pointer without alignment, or bytes without a pointer
    args = [None, P, P, P, P, P, 512, 256, 256, 512, None, None, 2, 3, 5, 4, 2, 128, 0.1]
    assert B.lib.rp_op_cross_attn_fwd(*args, P + 4, 64) == B.RP_EINVAL
    assert B.lib.rp_op_cross_attn_fwd(*args, None, 64) == B.RP_EINVAL


GOOD_BALANCE = [None, P, P, None, 8, 4, 16, 2, 0.1, 0.0, 1.0, P, P, P, None, P, P, 1 << 20]


@pytest.mark.parametrize("at,value", [(1, None), (2, None), (4, -1), (4, 6), (5, 0), (5, -4), (6, 0), (6, 1025), (7, 0), (7, 17), (11, None), (12, None), (13, None),
                                      (16, None), (16, P + 8), (17, 16)])
def test_balance_refuses(at, value):
    args = list(GOOD_BALANCE)
    args[at] = value
    assert B.lib.rp_op_moe_balance(*args) == B.RP_EINVAL


def test_balance_refuses_an_input_gradient_without_an_output():
    args = list(GOOD_BALANCE)
    args[14], args[15] = P, None
    assert B.lib.rp_op_moe_balance(*args) == B.RP_EINVAL
    for bad in ((-1, 4, 8), (6, 4, 8), (8, 0, 8), (8, 4, 0), (8, 4, 1025)):
        refused(B.rp_op_moe_balance_scratch, *bad)
    assert B.rp_op_moe_balance_scratch(0, 4, 8) == 0


def difference(f, x, direction, h=1e-6):
    return (f(x + h * direction) - f(x - h * direction)) / (2 * h)


def test_reference_gradients_against_differences():
    """The formulas that the kernels' gradients are tested with, against central differences in 64 bits (h = 1e-6: truncation
    1e-12 of the third derivative, rounding 1e-16 / 1e-6)."""
    g = torch.Generator().manual_seed(5)
    rnd = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    q, k, v, do = rnd(2, 5, 4, 8), rnd(2, 7, 2, 8), rnd(2, 7, 2, 8), rnd(2, 5, 4, 8)
    run = lambda q, k, v: R.cross_attention(q, k, v, do, [5, 3], [7, 4], 0.4, lambda n: True)  # noqa: E731
    got = run(q, k, v)
    for name, at in (("dq", 0), ("dk", 1), ("dv", 2)):
        x = [q, k, v]
        u = rnd(*x[at].shape)

        def value(t):
            y = list(x)
            y[at] = t
            return float((run(*y)["o"][0] * do).sum())

        want = float((got[name][0] * u).sum())
        assert abs(difference(value, x[at], u) - want) < 1e-7 * (1 + abs(want))
    logits, idx = rnd(12, 6), torch.stack([torch.randperm(6, generator=g)[:2] for _ in range(12)])
    mask = torch.tensor([1] * 9 + [0] * 3)
    loss = lambda x: float(R.balance(x, idx, mask, 4, 2, 0.7, 0.2, 1.0)[2][0])  # noqa: E731
    u = rnd(12, 6)
    want = float((R.balance(logits, idx, mask, 4, 2, 0.7, 0.2, 1.0)[3] * u).sum())
    assert abs(difference(loss, logits, u) - want) < 1e-8
    # the rotation's backward is its transpose: <R x, y> = <x, R^T y>
    th = R.frequencies(3, 1e4, 4.0, 1.0, 32.0, 64, 6)
    ang = torch.arange(9, dtype=torch.float64)[:, None] * th
    cs = torch.stack((ang.cos(), ang.sin()), -1)
    x, y = rnd(9, 3, 8), rnd(9, 3, 8)
    for layout in (0, 1):
        assert abs(float((R.rotate(x, cs, layout, 6, 0) * y).sum() - (x * R.rotate(y, cs, layout, 6, 1)).sum())) < 1e-12
