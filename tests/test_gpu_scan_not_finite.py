"""Infinities and NaN in the gated linear recurrence stay to the end of their document, also where the product of the gates on the way is too small for fp32."""
import pytest

from test_gpu_scan import B, Case, DEV  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BAD = [float("nan"), float("inf"), -float("inf")]


def small_gates(weight, n, begins, state=True):
    """Gates of sigmoid(-2): 16 of them 2^-49, 128 of them 2^-393; a document begins at `begins`."""
    c = Case(weight, 2, n, 72, state=state)
    c.g[:2 * n] = -2.0
    if begins:
        c.first = torch.zeros((2, n), dtype=torch.uint8, device=DEV)
        c.first[:, begins] = 1
    return c


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("weight", [0, 1, 2])
@pytest.mark.parametrize("n,begins", [(100, 0), (128, 77), (700, 0), (700, 515), (4500, 4100)])
def test_the_state_before(B, n, begins, weight, bad):  # noqa: F811
    plain = small_gates(weight, n, begins).run(B)
    want = {k: t.clone() for k, t in plain.got().items()}
    case = small_gates(weight, n, begins)
    case.h0[1, ::5] = bad
    got = case.run(B).got()
    end = begins or n
    spoiled = got["y"][1, :end, ::5]
    assert torch.equal(spoiled.isnan(), torch.full_like(spoiled, bad).isnan()) and bool((spoiled.isnan() | (spoiled == bad)).all())
    assert not bool(got["dg"][1, :end, ::5].isfinite().any())
    if not begins:
        assert not bool(got["last"][1, ::5].isfinite().any())
    rest = torch.ones(72, dtype=torch.bool, device=DEV)
    rest[::5] = False
    for name, t in got.items():      # nothing else has changed
        assert torch.equal(t[0], want[name][0]) and torch.equal(t[1][..., rest], want[name][1][..., rest]), name
        if begins and t.dim() == 3:
            assert torch.equal(t[1, begins:], want[name][1, begins:]), name


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("weight", [0, 1, 2])
@pytest.mark.parametrize("n,begins", [(100, 0), (128, 77), (700, 0), (700, 131), (4500, 300)])
def test_the_gradient_behind(B, n, begins, weight, bad):  # noqa: F811
    plain = small_gates(weight, n, begins).run(B)
    want = {k: t.clone() for k, t in plain.got().items()}
    case = small_gates(weight, n, begins)
    case.dlast[0, 1::7] = bad
    got = case.run(B).got()
    spoiled = got["dx"][0, begins:, 1::7]
    assert torch.equal(spoiled.isnan(), torch.full_like(spoiled, bad).isnan()) and bool((spoiled.isnan() | (spoiled == bad)).all())
    assert not bool(got["dg"][0, begins:, 1::7].isfinite().any())
    if not begins:
        assert not bool(got["dh0"][0, 1::7].isfinite().any())
    rest = torch.ones(72, dtype=torch.bool, device=DEV)
    rest[1::7] = False
    for name, t in got.items():
        assert torch.equal(t[1], want[name][1]) and torch.equal(t[0][..., rest], want[name][0][..., rest]), name
        if begins and t.dim() == 3:
            assert torch.equal(t[0, :begins], want[name][0, :begins]), name


@pytest.mark.parametrize("bad", BAD)
def test_a_token_between(B, bad):  # noqa: F811
    """An input and a gradient that are not finite, in the midst of a long sequence of two documents."""
    n, begins, at = 900, 600, 40
    case = small_gates(1, n, begins)
    case.x[at, 3] = bad
    case.dy[at, 3] = bad
    got = case.run(B).got()
    assert bool(got["y"][0, :at].isfinite().all()) and not bool(got["y"][0, at:begins, 3].isfinite().any()) and bool(got["y"][0, begins:].isfinite().all())
    assert not bool(got["dx"][0, :at + 1, 3].isfinite().any()) and bool(got["dx"][0, at + 1:].isfinite().all())
    assert not bool(got["dh0"][0, 3].isfinite().any()) and bool(got["last"].isfinite().all())
