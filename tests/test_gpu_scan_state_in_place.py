"""The gated linear recurrence with the state behind the last token written over the one before the first, and their gradients likewise: the bits of a call with an array for each."""
import pytest

from test_gpu_scan import B, Case  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("weight", [0, 1, 2])
@pytest.mark.parametrize("b,n,c,length", [(2, 100, 264, None), (3, 128, 72, [128, 0, 65]), (2, 300, 264, None), (3, 300, 72, [300, 0, 129]), (1, 2000, 1032, None), (2, 4500, 136, None)])
def test_last_in_the_place_of_h0(B, weight, b, n, c, length):  # noqa: F811
    """One chunk of tokens a sequence, several, and more than are looked back over at once."""
    apart = Case(weight, b, n, c, length=length).run(B).check()
    want = {k: t.clone() for k, t in apart.got().items()}
    case = Case(weight, b, n, c, length=length)
    case.last[:b * c] = case.h0.reshape(-1)
    case.h0 = case.last[:b * c].reshape(b, c)
    case.run(B)
    for name, t in case.got().items():
        assert torch.equal(t, want[name]), name


@pytest.mark.parametrize("weight", [0, 1, 2])
@pytest.mark.parametrize("b,n,c,length", [(2, 100, 264, None), (3, 128, 72, [128, 0, 65]), (3, 300, 72, [300, 0, 129]), (2, 4500, 136, None)])
def test_dh0_in_the_place_of_dlast(B, weight, b, n, c, length):  # noqa: F811
    want = {k: t.clone() for k, t in Case(weight, b, n, c, length=length).run(B).got().items()}
    case = Case(weight, b, n, c, length=length)
    case.dh0[:b * c] = case.dlast.reshape(-1)
    case.dlast = case.dh0[:b * c].reshape(b, c)
    case.run(B)
    for name, t in case.got().items():
        assert torch.equal(t, want[name]), name
