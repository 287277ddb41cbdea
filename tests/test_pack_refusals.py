"""What the operators for training on packed documents refuse, and their 64-bit references against differences.  Nothing is launched here."""
import math
import os

import pytest

import __graft_entry__
from paper_2604_27085_amd import build as _build
if not os.path.exists(_build.LIB):
    __graft_entry__.build()
from paper_2604_27085_amd import binding as B  # noqa: E402

import pack_reference as R  # noqa: E402

torch = pytest.importorskip("torch")
P = 4096      # an address that is never followed: every call below is refused before anything is enqueued


class Bytes:
    """Scratch of so many bytes at P."""

    def __init__(self, n, at=P):
        self.n, self.at = n, at

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.n

    def element_size(self):
        return 1


def refused(f, *args, code=B.RP_EINVAL, **kw):
    with pytest.raises(B.RpError) as e:
        f(*args, **kw)
    assert e.value.code == code


GOOD_SPAN = dict(q=P, k=P, v=P, o=P, o_rest=P, lse=P, ldq=512, ldk=256, ldv=256, ldo=512, span=P, q_pos=None, slopes=None, cap=0.0, batch=2, seq_q=3, seq_kv=5, a=4,
                 kh=2, d=128, scale=0.1)
BAD_SPAN = [dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(q=P + 8), dict(k=P + 2), dict(o_rest=P + 4), dict(ldq=508), dict(ldq=504), dict(ldk=248),
            dict(ldv=1 << 24), dict(ldk=0), dict(ldo=0), dict(span=None), dict(span=P + 4), dict(batch=-1), dict(seq_q=-1), dict(seq_kv=-1), dict(a=0), dict(kh=0),
            dict(kh=3), dict(d=96), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(cap=-1.0), dict(cap=math.nan), dict(cap=math.inf),
            dict(cap=1e-4), dict(cap=2e3), dict(seq_q=1 << 30), dict(seq_kv=1 << 30), dict(batch=1 << 30)]


@pytest.mark.parametrize("bad", BAD_SPAN)
def test_span_forward_refuses(bad):
    refused(B.rp_op_span_attn_fwd, None, **dict(GOOD_SPAN, **bad))


@pytest.mark.parametrize("bad", BAD_SPAN + [dict(dout=None), dict(lse=None), dict(delta=None), dict(dq=None), dict(dk=None), dict(dv=P + 8), dict(lddq=256),
                                            dict(lddo=500), dict(lddk=248), dict(lddv=1 << 24), dict(scratch=None), dict(scratch=Bytes(16)),
                                            dict(scratch=Bytes(1 << 20, P + 8))])
def test_span_backward_refuses(bad):
    good = dict(GOOD_SPAN, dout=P, delta=P, dq=P, dk=P, dv=P, lddo=512, lddq=512, lddk=256, lddv=256, scratch=Bytes(1 << 20))
    refused(B.rp_op_span_attn_bwd, None, **dict(good, **bad))


def test_span_scratch():
    with pytest.raises(B.RpError):
        B.rp_op_span_attn_scratch(1, 1, 1, 3, 2, 64)
    assert B.rp_op_span_attn_scratch(0, 0, 0, 4, 2, 64) == (0, 0, 0)
    assert B.rp_op_span_attn_scratch(64, 4096, 4096, 32, 32, 128)[0] == 0      # rows enough for the chip
    f, b, least = B.rp_op_span_attn_scratch(1, 1, 32768, 8, 8, 128)
    assert 0 < f and 16 + 8 * 256 <= least < b
    assert B.lib.rp_op_span_attn_scratch(1, 1, 32768, 8, 8, 128, None, None, None) == B.RP_OK
    assert B.rp_op_span_attn_scratch(3, 100, 7, 6, 2, 64)[2] == 512      # 16 bytes for 64 rows of a key head, 8 for 128 keys, each rounded up to 256
    refused(B.rp_op_span_attn_fwd, None, **dict(GOOD_SPAN, scratch=Bytes(64, P + 4)))


@pytest.mark.parametrize("batch,seq_q,seq_kv,d,backward", [(1 << 24, 1, 1, 64, 0), (1 << 23, 129, 1, 64, 0), (1 << 24, 1, 1, 64, 1), (1 << 23, 1, 1, 128, 1),
                                                           (1 << 22, 1, 129, 128, 1), (1 << 23, 1, 129, 64, 1)])
def test_span_refuses_more_blocks_than_a_launch_has(batch, seq_q, seq_kv, d, backward):
    args = dict(GOOD_SPAN, batch=batch, seq_q=seq_q, seq_kv=seq_kv, a=1, kh=1, d=d)
    if backward:
        refused(B.rp_op_span_attn_bwd, None, **dict(args, dout=P, delta=P, dq=P, dk=P, dv=P, lddo=512, lddq=512, lddk=256, lddv=256, scratch=Bytes(1 << 40)))
    else:
        refused(B.rp_op_span_attn_fwd, None, **args)


@pytest.mark.parametrize("bad", [dict(starts=None), dict(n_docs=-1), dict(window=-1), dict(T_=-1), dict(T_=(1 << 30) + 8), dict(seq=0), dict(seq=-8), dict(T_=12), dict(span=P + 4)])
def test_plan_refuses(bad):
    refused(B.rp_op_pack_plan, None, **dict(dict(starts=P, prefix=None, n_docs=2, window=0, T_=16, seq=8, span=P, pos=P, first=P), **bad))


GOOD_SCAN = dict(weight=1, x=P, g=P, ldx=64, ldg=64, first=None, len_=None, states=P, batch=2, seq=300, c=64, scratch=Bytes(1 << 20))
BAD_SCAN = [dict(weight=-1), dict(weight=3), dict(x=None), dict(g=None), dict(x=P + 2), dict(ldx=60), dict(ldx=56), dict(ldg=1 << 24), dict(states=P + 8), dict(batch=-1),
            dict(seq=-1), dict(c=-8), dict(c=60), dict(c=1 << 24), dict(seq=1 << 30), dict(batch=1 << 30), dict(scratch=None), dict(scratch=Bytes(64)),
            dict(scratch=Bytes(1 << 20, P + 4))]


@pytest.mark.parametrize("bad", BAD_SCAN + [dict(y=None), dict(y=P + 4), dict(ldy=8), dict(h0=P + 4), dict(last=P + 2)])
def test_scan_forward_refuses(bad):
    refused(B.rp_op_scan_fwd, None, **dict(dict(GOOD_SCAN, y=P, ldy=64, h0=None, last=None), **bad))


@pytest.mark.parametrize("bad", BAD_SCAN + [dict(states=None), dict(dy=None), dict(dx=None), dict(dg=P + 8), dict(lddy=60), dict(lddx=8), dict(lddg=1 << 24), dict(dlast=P + 4),
                                            dict(dh0=P + 8)])
def test_scan_backward_refuses(bad):
    refused(B.rp_op_scan_bwd, None, **dict(dict(GOOD_SCAN, dy=P, dx=P, dg=P, lddy=64, lddx=64, lddg=64, dlast=None, dh0=None), **bad))


@pytest.mark.parametrize("bad", [dict(dx=3 * P, x=3 * P, lddx=72), dict(dx=4 * P, dy=4 * P, lddx=72), dict(dg=5 * P, g=5 * P, lddg=72)])
def test_scan_backward_in_place_keeps_the_stride(bad):
    apart = dict(x=P, g=2 * P, dy=6 * P, dx=7 * P, dg=8 * P, lddy=64, lddx=64, lddg=64, dlast=None, dh0=None)
    refused(B.rp_op_scan_bwd, None, **dict(dict(GOOD_SCAN, **apart), **bad))


def test_scan_sizes():
    refused(B.rp_op_scan_sizes, 1, 1, 12)
    assert B.rp_op_scan_sizes(0, 9, 8) == (0, 0) and B.rp_op_scan_sizes(2, 0, 8) == (0, 0)
    assert B.rp_op_scan_sizes(8, 1, 4096)[1] == 0      # the step of a generation needs no scratch
    assert B.rp_op_scan_sizes(2, 129, 8)[0] == 2 * 2 * 8 * 4      # a state for 128 tokens
    assert B.lib.rp_op_scan_sizes(1, 1, 8, None, None) == B.RP_OK


GOOD_EMBED = dict(ids=P, scale=1.0, T_=100, V=50, h=64)
BAD_EMBED = [dict(ids=None), dict(scale=math.nan), dict(scale=math.inf), dict(T_=-1), dict(T_=1 << 24), dict(V=-1), dict(V=1 << 20), dict(h=60), dict(h=-8), dict(h=65544),
             dict(T_=(1 << 24) - 1, h=65536)]


@pytest.mark.parametrize("bad", BAD_EMBED + [dict(table=None), dict(table=P + 2), dict(ldt=56), dict(ldt=60), dict(x=None), dict(x=P + 8), dict(ldx=0)])
def test_embedding_refuses(bad):
    refused(B.rp_op_embed_fwd, None, **dict(dict(GOOD_EMBED, table=P, ldt=64, x=P, ldx=64), **bad))


@pytest.mark.parametrize("bad", BAD_EMBED + [dict(dx=None), dict(dx=P + 8), dict(lddx=8), dict(dtable=None), dict(dtable=P + 4), dict(lddt=60), dict(scratch=None),
                                             dict(scratch=Bytes(100)), dict(scratch=Bytes(1 << 20, P + 8))])
def test_embedding_gradient_refuses(bad):
    refused(B.rp_op_embed_bwd, None, **dict(dict(GOOD_EMBED, dx=P, lddx=64, dtable=P, lddt=64, accumulate=1, scratch=Bytes(1 << 20)), **bad))
    refused(B.rp_op_embed_scratch, 1, 1, 12)


@pytest.mark.parametrize("bad", [dict(x=None), dict(y=None), dict(x=P + 2), dict(y=P + 8, ldy=64), dict(res=P + 4), dict(ldx=60), dict(ldx=56), dict(ldy=1 << 24), dict(res=P, ldr=8),
                                 dict(T_=-1), dict(n=-8), dict(n=60), dict(p=-0.1), dict(p=1.1), dict(p=math.nan), dict(y=P, ldy=128), dict(res=2 * P, y=2 * P, ldr=72),
                                 dict(step=P + 4), dict(T_=1 << 30, n=1 << 20, ldx=1 << 20, ldy=1 << 20, ldr=1 << 20)])
def test_dropout_refuses(bad):
    refused(B.rp_op_dropout, None, **dict(dict(x=P, ldx=64, res=None, ldr=64, y=2 * P, ldy=64, T_=10, n=64, p=0.1, seed=1, offset=0, step=None), **bad))


# ---------------------------------------------------------------------------------------------------- the references
def difference(f, x, direction, h=1e-6):
    return (f(x + h * direction) - f(x - h * direction)) / (2 * h)


@pytest.mark.parametrize("cap,bias", [(0.0, False), (1.5, True)])
def test_attention_reference_against_differences(cap, bias):
    """Central differences in 64 bits (h = 1e-6: truncation 1e-12 of the third derivative, rounding 1e-16 / 1e-6)."""
    g = torch.Generator().manual_seed(5)
    rnd = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    q, k, v, do = rnd(2, 5, 4, 8), rnd(2, 7, 2, 8), rnd(2, 7, 2, 8), rnd(2, 5, 4, 8)
    span = torch.tensor([[[0, 7], [2, 3], [5, 4], [-2, 9], [1, 6]], [[0, 1], [0, 2], [1, 3], [3, 7], [6, 7]]])
    pos = torch.randint(0, 7, (2, 5), generator=g)
    slopes = torch.tensor([0.5, 0.25, 0.125, 1.0]) if bias else None
    run = lambda q, k, v: R.span_attention(q, k, v, do, span, pos, slopes, cap, 0.4)  # noqa: E731
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


@pytest.mark.parametrize("weight", [0, 1, 2])
def test_scan_reference_against_differences(weight):
    g = torch.Generator().manual_seed(6)
    rnd = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    x, gate, dy, h0, dlast = rnd(2, 9, 3), rnd(2, 9, 3), rnd(2, 9, 3), rnd(2, 3), rnd(2, 3)
    first = torch.zeros((2, 9), dtype=torch.uint8)
    first[0, 4] = first[1, 7] = 1
    length = [9, 6]
    on = torch.stack([torch.arange(9) < m for m in length])[..., None]
    run = lambda x, gate, h0: R.scan(weight, x, gate, dy, first, length, h0, dlast)  # noqa: E731
    got = run(x, gate, h0)
    for name, at in (("dx", 0), ("dg", 1), ("dh0", 2)):
        ins = [x, gate, h0]
        u = rnd(*ins[at].shape)

        def value(t):
            y = list(ins)
            y[at] = t
            r = run(*y)
            return float((r["y"][0] * dy * on).sum() + (r["last"][0] * dlast).sum())

        want = float((got[name][0] * u).sum())
        assert abs(difference(value, ins[at], u) - want) < 1e-8 * (1 + abs(want))


def test_generator_against_the_published_vectors():
    """Philox 4x32-10: counter and key of zeros, of ones, and of the digits of pi, as published with the generator."""
    assert R.philox([0, 0, 0, 0], [0, 0]) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    m = 0xFFFFFFFF
    assert R.philox([m, m, m, m], [m, m]) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert R.philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]
