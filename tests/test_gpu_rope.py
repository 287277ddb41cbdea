"""Rotary positions in both pair layouts, over part of a head, at given positions, and their scaled tables, against 64-bit formulas."""
import math

import numpy as np
import pytest

import ops_reference as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_27085_amd import binding
    return binding


def stream():
    return torch.cuda.current_stream().cuda_stream


TABLES = [(0, 1.0e6, 1.0, 1.0, 1000, 128), (1, 1.0e4, 4.0, 1.0, 515, 64), (2, 5.0e5, 8.0, 1.0, 77, 96), (3, 1.0e6, 32.0, 1.25, 3001, 128), (3, 1.0e4, 2.0, 1.0, 1, 2),
          (0, 1.0e4, 1.0, 1.0, 9, 512), (3, 1.0e6, 40.0, 1.0, 1 << 20, 6), (1, 1.0e4, 4.0, -2.0, 20000, 34), (0, 1.0e4, 1.0, 1.0, 5, 2)]


@pytest.mark.parametrize("kind,base,factor,amplitude,n_pos,rot", TABLES)
def test_table(B, kind, base, factor, amplitude, n_pos, rot):
    """Half a step of fp32 (2^-24 of the value), and the angle's rounding: p theta / 2 pi in 64 bits is off by 2^-52 of it, below 2^20 / 6
    turns 4e-11 turns or 3e-10 rad; the polynomials 1e-11 (numpy's own 64-bit angle is as far off)."""
    guard = 64
    buf = torch.full((n_pos * rot + guard,), float("nan"), dtype=torch.float32, device=DEV)
    B.rp_op_rope_table_scaled(stream(), buf, B.make_rope_scaling(kind, base, factor, 1.0, 32.0, 4096, amplitude), n_pos, rot)
    torch.cuda.synchronize()
    assert bool(torch.isnan(buf[n_pos * rot:]).all())
    got = buf[:n_pos * rot].reshape(n_pos, rot // 2, 2).cpu().double()
    ang = torch.arange(n_pos, dtype=torch.float64)[:, None] * R.frequencies(kind, base, factor, 1.0, 32.0, 4096, rot)
    amp = float(np.float32(amplitude))
    want = amp * torch.stack((ang.cos(), ang.sin()), -1)
    assert bool(((got - want).abs() <= 2.0 ** -24 * want.abs() + 2.0e-9 * abs(amp)).all())


def test_table_is_what_the_normed_rotation_takes(B):
    """rp_op_qknorm_rope on a plain scaled table: the same angles as rp_op_rope_table's, up to one rounding of each."""
    a = torch.empty((300, 64, 2), dtype=torch.float32, device=DEV)
    b = torch.empty_like(a)
    B.rp_op_rope_table(stream(), a, 300, 128, 1.0e6)
    B.rp_op_rope_table_scaled(stream(), b, B.make_rope_scaling(0, 1.0e6), 300, 128)
    torch.cuda.synchronize()
    assert float((a - b).abs().max()) <= 2.0 ** -23


CASES = [
    # layout, d, rot, a, k, T, seq, positions
    (0, 128, 128, 16, 8, 7, 7, None), (1, 128, 128, 16, 8, 7, 7, "given"), (0, 64, 32, 5, 1, 301, 301, "given"), (1, 64, 32, 5, 1, 301, 43, None),
    (0, 96, 24, 3, 3, 130, 65, None), (0, 96, 12, 3, 2, 33, 33, None), (0, 80, 6, 2, 2, 50, 25, "given"), (1, 80, 6, 2, 2, 50, 25, "given"), (0, 64, 2, 1, 1, 4, 2, None),
    (1, 8, 8, 1, 0, 1, 1, None), (0, 16, 16, 0, 2, 3, 3, None), (1, 512, 512, 2, 1, 5, 5, None), (0, 512, 500, 2, 1, 5, 5, "given"), (0, 128, 64, 64, 8, 1021, 1021, None),
    (1, 256, 64, 71, 9, 100, 100, "given"), (1, 72, 70, 4, 4, 19, 19, None), (0, 72, 70, 4, 4, 19, 19, None),
]


@pytest.mark.parametrize("bwd", [0, 1])
@pytest.mark.parametrize("how", ["dense", "strided", "in place"])
@pytest.mark.parametrize("layout,d,rot,a,k,T,seq,given", CASES)
def test_rotation(B, layout, d, rot, a, k, T, seq, given, how, bwd):
    """Two products and a sum in fp32 (4 * 2^-24 of |x| + |y|), then half a step of bf16; what is not turned is the same bits."""
    g = torch.Generator().manual_seed(T * 1000 + d + rot + layout)
    n_pos = 50 if given else seq
    n_pos = max(n_pos, seq)
    pos = torch.randint(0, n_pos, (T,), generator=g, dtype=torch.int32) if given else torch.arange(T, dtype=torch.int32) % seq
    cs = torch.randn((n_pos, rot // 2, 2), generator=g)
    pad = 0 if how == "dense" else 16
    width = (a + k) * d + pad
    src = torch.randn((T, width), generator=g).to(torch.bfloat16)
    dev_in = src.to(DEV)
    dev_out = dev_in if how == "in place" else torch.full((T, width), float("nan"), dtype=torch.bfloat16, device=DEV)
    heads = lambda t, lo, n: t[:, lo:lo + n * d].reshape(T, n, d)  # noqa: E731
    off = pad // 2      # (8 elements: 16 bytes)
    q0, k0 = off, off + a * d
    args = lambda t: (t[:, q0:] if a else None, t[:, k0:] if k else None, width, width)  # noqa: E731
    B.rp_op_rope(stream(), bwd, layout, d, rot, *args(dev_in), *args(dev_out), cs.to(DEV), n_pos, pos.to(DEV) if given else None, T, seq, a, k)
    torch.cuda.synchronize()
    got = dev_out.cpu()
    for lo, n in ((q0, a), (k0, k)):
        if not n:
            continue
        x, y = heads(src, lo, n), heads(got, lo, n)
        want = R.rotate(x, cs[pos.long()], layout, rot, bwd)
        c = cs[pos.long()].abs()
        size = R.rotate(x.abs(), c, layout, rot, 0).abs() + R.rotate(x.abs(), c, layout, rot, 1).abs()      # |x c| + |y s| or more
        bound = 2.0 ** -8 * want.abs() + 2.0 ** -21 * size + 1e-30
        assert bool(((y.double() - want).abs() <= bound)[..., :rot].all())
        assert bool(torch.equal(y[..., rot:], x[..., rot:]))
    # the columns beside the heads stay as they were
    if pad:
        want = src if how == "in place" else torch.full_like(src, float("nan"))
        for sl in (slice(0, off), slice(off + (a + k) * d, width)):
            assert torch.equal(got[:, sl].view(torch.int16), want[:, sl].view(torch.int16))


def test_positions_without_a_row_become_nan(B):
    d, rot, T = 64, 32, 6
    x = torch.randn((T, 2, d), device=DEV).to(torch.bfloat16)
    out = torch.zeros_like(x)
    pos = torch.tensor([0, 9, 10, -1, 2 ** 31 - 1, 3], dtype=torch.int32, device=DEV)
    cs = torch.ones((10, rot // 2, 2), device=DEV)
    for layout in (0, 1):
        B.rp_op_rope(stream(), 0, layout, d, rot, x, None, 2 * d, 0, out, None, 2 * d, 0, cs, 10, pos, T, 1, 2, 0)
        torch.cuda.synchronize()
        nan = torch.isnan(out)
        assert nan[2:5, :, :rot].all() and not nan[[0, 1, 5]].any() and not nan[..., rot:].any()
        assert torch.equal(out[..., rot:], x[..., rot:])


def test_nothing_to_do(B):
    B.rp_op_rope_table_scaled(stream(), None, B.make_rope_scaling(), 0, 64)
    B.rp_op_rope(stream(), 0, 0, 64, 64, None, None, 128, 64, None, None, 128, 64, None, 0, None, 0, 1, 2, 1)
    x = torch.randn((4, 64), device=DEV).to(torch.bfloat16)
    B.rp_op_rope(stream(), 0, 0, 64, 64, None, None, 0, 0, None, None, 0, 0, torch.ones((4, 32, 2), device=DEV), 4, None, 4, 4, 0, 0)
    torch.cuda.synchronize()
    assert math.isfinite(float(x.float().sum()))
