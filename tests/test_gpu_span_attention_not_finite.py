"""Infinities and NaN that a query does see, in one of q, k, v and the gradient of o alone: whatever of dq, dk, dv the formulas make not finite of them shows, row by row, and nothing that
does not see them changes by a bit."""
import pytest

import pack_reference as R
from test_gpu_span_attention import B, Case, DEV, I32  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
INF, NAN = float("inf"), float("nan")
HEADS = [(4, 2, 64), (6, 2, 64), (4, 2, 128), (6, 2, 128)]      # groups that divide a tile of 64 rows, and that do not
SIZES = [(300, 90, 171), (850, 190, 755)]                       # dS in two parts and in one; documents of tiles at their edges alone, and of whole ones too
KINDS = [(0.0, False), (20.0, False), (20.0, True)]


def make(size, heads, kind):
    T, lo, hi = size
    c = Case("causal", 1, T, T, *heads, cap=kind[0], bias=kind[1])
    c.span.copy_(torch.tensor(R.plan([0, lo, hi, T], None, 0, T, T)[0], dtype=I32))
    return c


def spoilt(t):      # [1, n, heads, d] -> [n, heads]
    return ~t[0].isfinite().all(-1)


def shows(got, want, name, rows, heads, at_least=True):
    """The rows x heads are not finite, the others the bits of the clean run."""
    bad = torch.zeros(got[name].shape[1:3], dtype=torch.bool, device=DEV)
    bad[rows[:, None], torch.tensor(heads, device=DEV)] = True
    if at_least:
        assert bool(spoilt(got[name])[bad].all()), name
    assert torch.equal(got[name][0][~bad], want[name][0][~bad]), name


def places(size):      # rows of the middle document: at its beginning, its end, and in between
    T, lo, hi = size
    return [lo, lo + 1, (lo + hi) // 2, hi - 1]


@pytest.mark.parametrize("scratch", ["full", "least"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("size", SIZES)
def test_gradient_of_o(B, size, heads, kind, scratch):  # noqa: F811
    a, kh, d = heads
    T, lo, hi = size
    want = make(size, heads, kind).run(B, scratch).got()
    every = torch.arange(T, device=DEV)
    for at, bad in zip(places(size), (INF, NAN, -INF, INF)):
        c = make(size, heads, kind)
        head = a - 1
        c.do[at, head * d + 5] = bad
        got = c.run(B, scratch).got()
        keys = every[(every >= lo) & (every <= at)]
        assert torch.equal(got["o"], want["o"]) and torch.equal(got["lse"], want["lse"])
        shows(got, want, "dq", every[at:at + 1], [head])
        shows(got, want, "dk", keys, [kh - 1])
        shows(got, want, "dv", keys, [kh - 1])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("size", SIZES)
def test_q(B, size, heads, kind):  # noqa: F811
    """Under a cap an infinite q has finite scores, an o and an lse; dk, which is dS times q, is not finite all the same."""
    a, kh, d = heads
    T, lo, hi = size
    want = make(size, heads, kind).run(B).got()
    every = torch.arange(T, device=DEV)
    for at, bad in zip(places(size), (INF, -INF, INF, NAN)):
        c = make(size, heads, kind)
        c.q[at, 7] = bad      # (of head 0)
        got = c.run(B).got()
        keys = every[(every >= lo) & (every <= at)]
        if bad != bad or not kind[0]:
            assert bool(spoilt(got["o"])[at, 0]) and bool(spoilt(got["dq"])[at, 0]) and bool(spoilt(got["dv"])[keys, 0].all())
        shows(got, want, "o", every[at:at + 1], [0], False)
        shows(got, want, "dq", every[at:at + 1], [0], False)
        shows(got, want, "dk", keys, [0])
        shows(got, want, "dv", keys, [0], False)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("size", SIZES)
def test_k(B, size, heads, kind):  # noqa: F811
    """A key of infinities that no query has any weight on, or under a cap some: o is finite, and dq, which is dS times k, is not."""
    a, kh, d = heads
    T, lo, hi = size

    def case():
        c = make(size, heads, kind)
        c.q[:T, 3::d] = c.q[:T, 3::d].abs() + 0.5      # so that the scores of the key are -inf, or -cap
        return c

    want = case().run(B).got()
    every = torch.arange(T, device=DEV)
    for at in places(size)[1:]:
        c = case()
        c.k[at, (kh - 1) * d + 3] = -INF
        got = c.run(B).got()
        rows = every[(every >= at) & (every < hi)]
        mine = list(range(a // kh * (kh - 1), a))
        assert bool(got["o"].isfinite().all()) and bool(got["lse"].isfinite().all())
        shows(got, want, "dq", rows, mine)
        if not kind[0]:      # no weight on it: it gets no gradient
            assert bool((got["dk"][0, at, kh - 1] == 0).all()) and bool((got["dv"][0, at, kh - 1] == 0).all())
        keys = every[(every >= lo) & (every < hi)]
        shows(got, want, "dk", keys, [kh - 1], False)
        shows(got, want, "dv", keys, [kh - 1], False)


@pytest.mark.parametrize("bad", [INF, NAN])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("size", SIZES)
def test_v(B, size, heads, kind, bad):  # noqa: F811
    """P does not know of v: lse and dv, which is P times the gradient of o, keep their bits."""
    a, kh, d = heads
    T, lo, hi = size
    want = make(size, heads, kind).run(B).got()
    every = torch.arange(T, device=DEV)
    for at in places(size):
        c = make(size, heads, kind)
        c.v[at, 11] = bad
        got = c.run(B).got()
        rows = every[(every >= at) & (every < hi)]
        mine = list(range(a // kh))
        assert torch.equal(got["lse"], want["lse"]) and torch.equal(got["dv"], want["dv"])
        shows(got, want, "o", rows, mine)
        shows(got, want, "dq", rows, mine)
        shows(got, want, "dk", every[(every >= lo) & (every < hi)], [0])


@pytest.mark.parametrize("kind", [(0.0, False), (0.0, True)])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("size", SIZES)
def test_a_query_whose_scores_are_all_minus_infinity(B, size, heads, kind):  # noqa: F811
    """The first query of a document whose only key is infinite: 0 / 0 in every weight."""
    a, kh, d = heads
    T, lo, hi = size
    c = make(size, heads, kind)
    c.q[:T, 3::d] = c.q[:T, 3::d].abs() + 0.5
    c.k[lo, 3::d] = -INF
    got = c.run(B).got()
    for name in ("o", "dq", "dk", "dv"):
        assert bool(spoilt(got[name])[lo].all()), name
    assert bool(got["o"][0, lo + 1:hi].isfinite().all())
    for name in ("o", "dq", "dk", "dv"):
        assert bool(got[name][0, :lo].isfinite().all()) and bool(got[name][0, hi:].isfinite().all()), name


@pytest.mark.parametrize("scratch", ["full", "least"])
@pytest.mark.parametrize("bad", [INF, NAN])
@pytest.mark.parametrize("kind,b,nq,nk,a,kh,d", [("all", 1, 1, 4096, 8, 8, 128), ("ragged", 2, 3, 3000, 8, 2, 64), ("all", 1, 150, 2048, 4, 4, 64), ("causal", 1, 150, 2500, 4, 4, 128)])
def test_v_of_keys_without_weight(B, kind, b, nq, nk, a, kh, d, bad, scratch):  # noqa: F811
    """0 times what is not finite, in a slice of the keys (or a call in one) that has no weight at all: NaN in o, and in what o is made of alone."""
    c = Case(kind, b, nq, nk, a, kh, d)
    c.q[:b * nq] = c.q[:b * nq].abs() + 0.5
    c.k[:nk - 40, 3::d] = -INF      # the scores of all keys of the first sequence but its last 40 are -inf
    want = {n: t.clone() for n, t in c.run(B, scratch, backward=False).got().items()}
    some = c.span[0, :, 1] > nk - 40      # (a causal query may see none of those: -inf throughout, 0 / 0)
    assert bool(some.any()) and bool(want["o"][0, some].isfinite().all()) and bool(want["lse"][0, :, some].isfinite().all()) and bool(want["o"][0, ~some].isnan().all())
    c.v[77, d + 5] = bad            # (of key head 1)
    got = c.run(B, scratch, backward=False).got()
    assert torch.equal(got["lse"], want["lse"])
    mine = list(range(a // kh, 2 * (a // kh)))
    assert bool(got["o"][0, :, mine, 5].isnan().all())
    others = [h for h in range(a) if h not in mine]
    assert torch.equal(got["o"][0, some][:, others], want["o"][0, some][:, others]) and torch.equal(got["o"][1:], want["o"][1:])
