"""What the accuracy limits of cross attention's gradients tell apart, on a 64-bit model of the kernels' roundings: the kernels' way stays inside them, each
step of it left out does not."""
import math

import pytest

import attention_accuracy as A

torch = pytest.importorskip("torch")


def inputs(rows, n, d, gain=None, std=2.0, seed=0):
    g = torch.Generator().manual_seed(seed + n + d)
    k, v, do = [torch.randn((m, h, d), generator=g).to(torch.bfloat16) for m, h in ((n, 1), (n, 1), (rows, 2))]
    q = A.sharp_queries(k.float(), 2, rows, gain, g) if gain else std * torch.randn((rows, 2, d), generator=g)
    return q.to(torch.bfloat16), k, v, do


def inside(got, want, name):
    value, bound = want[name]
    return bool(((got[name] - value).abs() <= bound).all())


def run(x, d, exact=False, **kw):
    return A.as_the_kernels_round(*x, d ** -0.5, exact, **kw), A.gradients(*x, d ** -0.5, exact)


def test_one_rounding():
    x = torch.randn(1 << 20, dtype=torch.float64, generator=torch.Generator().manual_seed(1))
    assert abs(A.distance(A.bf16(x), x) - A.ONE_ROUNDING) < 0.02e-3


@pytest.mark.parametrize("n,d,exact,std", [(128, 128, True, 1.0), (128, 64, True, 2.0), (129, 128, False, 1.0), (700, 128, True, 2.0), (1500, 64, False, 1.0)])
def test_ordinary_rows(n, d, exact, std):
    x = inputs(400, n, d, std=std)
    got, want = run(x, d, exact)
    assert A.distance(got["dq"], want["dq"][0]) < A.DQ_ORDINARY
    assert inside(got, want, "dq") and inside(got, want, "dk")
    one, _ = run(x, d, exact, parts=1)
    assert A.distance(one["dq"], want["dq"][0]) > A.DQ_ORDINARY      # dS in one part


@pytest.mark.parametrize("gain", [1.0, 1.2])
@pytest.mark.parametrize("n,d", [(129, 128), (700, 128), (1500, 128), (700, 64)])
def test_sharp_rows(n, d, gain):
    gain *= math.sqrt(128.0 / d)
    x = inputs(400, n, d, gain)
    got, want = run(x, d)
    assert A.distance(got["dq"], want["dq"][0]) < A.DQ_SHARP and A.distance(got["dk"], want["dk"][0]) < A.DK_SHARP
    assert inside(got, want, "dq") and inside(got, want, "dk")
    bad, _ = run(x, d, repeat=False)      # the stored output's delta for dq
    assert A.distance(bad["dq"], want["dq"][0]) > 2 * A.DQ_SHARP and not inside(bad, want, "dq")
    bad, _ = run(x, d, correct=False)     # and for dk
    assert A.distance(bad["dk"], want["dk"][0]) > A.DK_SHARP and not inside(bad, want, "dk")
    got, want = run(x, d, True)
    assert A.distance(got["dq"], want["dq"][0]) < A.DQ_SHARP_EXACT
    assert inside(got, want, "dq") and inside(got, want, "dk")


@pytest.mark.parametrize("share", [1.0, 3.0])
@pytest.mark.parametrize("n,d", [(300, 128), (705, 64)])
def test_keys_that_share_a_part(n, d, share):
    q, k, v, do = inputs(400, n, d, std=1.0)
    k = (k.float() + share * torch.randn((1, 1, d), generator=torch.Generator().manual_seed(n))).to(torch.bfloat16)
    got, want = run((q, k, v, do), d)
    assert A.distance(got["dq"], want["dq"][0]) < A.DQ_ORDINARY and inside(got, want, "dq")
    bad, _ = run((q, k, v, do), d, repeat=False)
    assert A.distance(bad["dq"], want["dq"][0]) > A.DQ_ORDINARY
