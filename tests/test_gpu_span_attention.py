"""Attention with a span of keys for every query, forward and backward, against 64-bit attention with bounds counted from its roundings (pack_reference)."""
import pytest

import pack_reference as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
BF16, I32 = torch.bfloat16, torch.int32
NAN = float("nan")


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_27085_amd import binding
    return binding


def spans(kind, b, nq, nk, g):
    """[b, nq, 2] and positions [b, nq]."""
    t = torch.arange(nq)
    pos = (t + nk - nq).expand(b, nq)
    if kind == "causal":
        return torch.stack((torch.zeros_like(pos), pos + 1), -1), pos
    if kind == "all":
        return torch.stack((torch.zeros_like(pos), torch.full_like(pos, nk)), -1), pos
    if kind == "docs":          # documents, the first part of each seeing itself both ways, windows, padding behind the last
        cuts = sorted(torch.randint(0, max(nq, 1), (4,), generator=g).tolist())
        starts = [0] + cuts[:3] + [cuts[3]]
        prefix = [5, 0, 40, 7]
        sp = R.plan(starts, prefix, 37, nq, nq)[0]
        return torch.tensor(sp).expand(b, nq, 2), pos
    if kind == "ragged":        # caches of lengths of their own, one of them empty
        n = torch.randint(nq, nk + 1, (b, 1), generator=g)
        n[0] = nk
        pos = n - nq + t
        sp = torch.stack((torch.zeros_like(pos), pos + 1), -1)
        if b > 1:
            sp[1] = 0
        return sp, pos
    lo = torch.randint(-5, nk + 5, (b, nq), generator=g)      # "any": also empty, reversed, beyond both ends, and in no order
    hi = lo + torch.randint(-3, max(nk // 2, 2), (b, nq), generator=g)
    return torch.stack((lo, hi), -1), torch.randint(0, nk + 1, (b, nq), generator=g)


class Case:
    """Inputs and outputs inside larger arrays: `pad` columns beside the heads and two rows behind the last sequence, all of them NaN, as the outputs are before the calls."""

    def __init__(self, kind, b, nq, nk, a, kh, d, cap=0.0, bias=False, pad=0, seed=0, std=2.0, rest=True, given_pos=True):
        self.shape, self.cap, self.pad = (b, nq, nk, a, kh, d), cap, pad
        g = torch.Generator().manual_seed(seed + 7 * nq + 11 * nk + a + d)
        sp, pos = spans(kind, b, nq, nk, g)
        self.span, self.pos = sp.to(I32).contiguous().to(DEV), pos.to(I32).contiguous().to(DEV)
        self.given_pos = given_pos
        self.slopes = (2.0 ** -torch.arange(1, a + 1).float()).to(DEV) if bias else None

        def array(n, heads, std):
            t = torch.full((b * n + 2, heads * d + 2 * pad), NAN, dtype=BF16)
            if std:
                t[:b * n, pad:pad + heads * d] = (std * torch.randn((b * n, heads * d), generator=g)).to(BF16)
            return t.to(DEV)

        self.q, self.do, self.k, self.v = array(nq, a, std), array(nq, a, 1.0), array(nk, kh, 1.0), array(nk, kh, 1.0)
        self.o, self.rest, self.dq, self.dk, self.dv = array(nq, a, 0), array(nq, a, 0) if rest else None, array(nq, a, 0), array(nk, kh, 0), array(nk, kh, 0)
        nan = lambda: torch.full((b * a * nq + 16,), NAN, device=DEV)  # noqa: E731
        self.lse, self.delta = nan(), nan()
        self.scale = d ** -0.5

    def view(self, t, n):
        b, _, _, _, _, d = self.shape
        return t[:b * n, self.pad:t.shape[1] - self.pad].reshape(b, n, (t.shape[1] - 2 * self.pad) // d, d)

    def run(self, B, scratch="full", backward=True, lse=True, stream=None):
        b, nq, nk, a, kh, d = self.shape
        st = stream or torch.cuda.current_stream().cuda_stream
        fwd, bwd, least = B.rp_op_span_attn_scratch(b, nq, nk, a, kh, d)
        size = {"full": (fwd, bwd), "least": (0, least), "some": (fwd // 2, least + (bwd - least) // 2)}[scratch]
        ws = [torch.full(((n + 3) // 4,), NAN, device=DEV) if n else None for n in size]
        at = lambda t: t.data_ptr() + 2 * self.pad if t is not None else None  # noqa: E731
        ld = lambda t: t.shape[1]  # noqa: E731
        pos = self.pos if self.given_pos else None
        B.rp_op_span_attn_fwd(st, at(self.q), at(self.k), at(self.v), at(self.o), at(self.rest), self.lse if lse else None, ld(self.q), ld(self.k), ld(self.v),
                              ld(self.o), self.span, pos, self.slopes, self.cap, b, nq, nk, a, kh, d, self.scale, ws[0])
        if backward:
            B.rp_op_span_attn_bwd(st, at(self.q), at(self.k), at(self.v), at(self.o), at(self.rest), at(self.do), self.lse, self.delta, at(self.dq), at(self.dk),
                                  at(self.dv), ld(self.q), ld(self.k), ld(self.v), ld(self.o), ld(self.do), ld(self.dq), ld(self.dk), ld(self.dv), self.span, pos,
                                  self.slopes, self.cap, b, nq, nk, a, kh, d, self.scale, ws[1])
        torch.cuda.synchronize()
        return self

    def got(self):
        b, nq, nk, a, kh, d = self.shape
        return {"o": self.view(self.o, nq), "lse": self.lse[:b * a * nq].reshape(b, a, nq), "dq": self.view(self.dq, nq), "dk": self.view(self.dk, nk),
                "dv": self.view(self.dv, nk)}

    def want(self):
        b, nq, nk, a, kh, d = self.shape
        return R.span_attention(self.view(self.q, nq), self.view(self.k, nk), self.view(self.v, nk), self.view(self.do, nq), self.span, self.pos, self.slopes,
                                self.cap, self.scale, self.rest is not None)

    def check(self, backward=True, names=None):
        want, got = self.want(), self.got()
        for name in names or (("o", "lse") + (("dq", "dk", "dv") if backward else ())):
            value, bound = want[name]
            x = got[name].double()
            if name == "lse":
                assert torch.equal(torch.isneginf(x), torch.isneginf(value)), name
                fine = ~torch.isneginf(value)
                x, value, bound = x[fine], value[fine], bound[fine]
            assert bool(torch.isfinite(x).all()), name
            off = ((x - value).abs() / (bound + 1e-30))
            assert not off.numel() or float(off.max()) <= 1.0, (name, float(off.max()))
        b, nq, nk, a, kh, d = self.shape
        for t, n, heads in ((self.o, nq, a), (self.dq, nq, a), (self.dk, nk, kh), (self.dv, nk, kh)):      # nothing beside, nothing behind
            inside = torch.zeros_like(t, dtype=torch.bool)
            inside[:b * n, self.pad:self.pad + heads * d] = True
            assert bool(t[~inside].isnan().all())
        assert bool(self.lse[b * a * nq:].isnan().all()) and bool(self.delta[b * a * nq:].isnan().all())
        return self


SHAPES = [
    ("causal", 1, 300, 300, 4, 2, 64), ("causal", 2, 129, 129, 8, 8, 128), ("docs", 1, 517, 517, 6, 2, 64), ("docs", 2, 260, 260, 16, 1, 128), ("any", 2, 77, 200, 4, 4, 64),
    ("any", 1, 200, 77, 12, 4, 128), ("any", 3, 65, 640, 8, 2, 128), ("ragged", 3, 1, 700, 16, 2, 128), ("ragged", 2, 5, 70, 4, 2, 64), ("all", 1, 64, 64, 2, 1, 64),
    ("all", 1, 1, 1, 1, 1, 128), ("causal", 1, 1, 1, 4, 2, 64), ("any", 1, 1, 3000, 4, 2, 64), ("causal", 1, 40, 1500, 32, 8, 64),
    ("causal", 1, 33, 33, 96, 1, 64), ("any", 1, 20, 150, 64, 1, 128), ("any", 2, 30, 400, 10, 2, 128), ("docs", 1, 40, 40, 71, 1, 128),
]
KINDS = [(0.0, False), (20.0, False), (0.0, True), (3.0, True)]


@pytest.mark.parametrize("cap,bias", KINDS)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_forward_and_backward(B, shape, cap, bias):
    Case(*shape, cap=cap, bias=bias).run(B).check()


LONG = [("docs", 1, 700, 700, 6, 2, 128), ("causal", 2, 600, 600, 8, 2, 128), ("docs", 1, 900, 900, 8, 2, 64), ("any", 1, 550, 777, 6, 2, 64), ("any", 2, 300, 1030, 4, 1, 128),
        ("ragged", 2, 130, 1300, 10, 2, 64)]      # (beyond what dS of few keys goes through in two parts)


@pytest.mark.parametrize("scratch", ["full", "least"])
@pytest.mark.parametrize("cap,bias", KINDS)
@pytest.mark.parametrize("shape", LONG, ids=lambda s: "-".join(map(str, s)))
def test_more_keys(B, shape, cap, bias, scratch):
    Case(*shape, cap=cap, bias=bias, pad=8).run(B, scratch).check()


@pytest.mark.parametrize("bad", [NAN, float("inf")])
@pytest.mark.parametrize("a,kh,d,cap,bias", [(4, 2, 64, 0.0, False), (6, 2, 64, 20.0, True), (4, 2, 128, 20.0, True), (6, 2, 128, 0.0, False)])
def test_a_document_does_not_reach_another_of_many_keys(B, bad, a, kh, d, cap, bias):
    T, lo, hi = 850, 190, 555
    runs = []
    for spoil in (False, True):
        c = Case("causal", 1, T, T, a, kh, d, cap=cap, bias=bias)
        c.span.copy_(torch.tensor(R.plan([0, lo, hi, T], None, 0, T, T)[0], dtype=I32))
        if spoil:
            for t in (c.q, c.k, c.v, c.do):
                t[lo:hi:3, ::5] = bad
        runs.append(c.run(B).got())
    for name, t in runs[1].items():
        rows = torch.arange(T, device=DEV)
        keep = (rows < lo) | (rows >= hi)
        x, y = (r[name][:, :, keep] if name == "lse" else r[name][:, keep] for r in runs)
        assert torch.equal(x, y), name


@pytest.mark.parametrize("scratch", ["least", "some"])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[6], SHAPES[7], SHAPES[12]], ids=lambda s: "-".join(map(str, s)))
def test_less_scratch(B, shape, scratch):
    Case(*shape, cap=20.0, bias=True).run(B, scratch).check()


def test_strides_positions_and_optional_outputs(B):
    Case("docs", 1, 150, 150, 4, 2, 64, pad=8, bias=True).run(B).check()
    Case("any", 2, 150, 90, 4, 2, 128, pad=16).run(B).check()
    Case("causal", 1, 70, 190, 4, 2, 64, bias=True, given_pos=False).run(B).check()
    Case("causal", 1, 130, 130, 4, 2, 128, rest=False).run(B).check()
    c = Case("docs", 1, 150, 150, 4, 2, 64, rest=False).run(B, backward=False, lse=False)
    c.check(backward=False, names=("o",))
    assert bool(c.lse.isnan().all())


@pytest.mark.parametrize("scratch", ["all", "least"])
@pytest.mark.parametrize("a,kh,d", [(4, 2, 64), (6, 2, 128), (4, 1, 128)])
def test_key_tiles_of_two_documents(B, a, kh, d, scratch):
    """Documents that begin inside a key tile, the last one long: the row tiles of such a key tile are masked all along, and several workgroups share them."""
    T = 3001
    c = Case("causal", 1, T, T, a, kh, d)
    c.span.copy_(torch.tensor(R.plan([0, 3, 700, 1301, T], None, 0, T, T)[0], dtype=I32))
    c.run(B, *([] if scratch == "all" else [scratch])).check()


@pytest.mark.parametrize("b,nq,nk", [(0, 5, 5), (2, 0, 5), (2, 5, 0), (1, 0, 0)])
def test_empty(B, b, nq, nk):
    c = Case("any", b, nq, nk, 4, 2, 64).run(B)
    g = c.got()
    for name in ("o", "dq", "dk", "dv"):
        assert bool((g[name] == 0).all())
    assert bool(torch.isneginf(g["lse"]).all())


def test_no_query_sees_anything(B):
    for d in (64, 128):
        c = Case("causal", 2, 150, 150, 4, 2, d)
        c.span.zero_()
        c.run(B)
        g = c.got()
        for name in ("o", "dq", "dk", "dv"):
            assert bool((g[name] == 0).all())
        assert bool(torch.isneginf(g["lse"]).all())


@pytest.mark.parametrize("bad", [NAN, float("inf"), -float("inf")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, True)])
def test_a_document_does_not_reach_another(B, bad, d, cap, bias):
    """The middle one of three documents full of infinities or NaN: the others' numbers are the same bits as with ordinary ones there."""
    T, lo, hi = 300, 90, 171
    make = lambda: Case("causal", 1, T, T, 4, 2, d, cap=cap, bias=bias)  # noqa: E731
    runs = []
    for spoil in (False, True):
        c = make()
        c.span.copy_(torch.tensor(R.plan([0, lo, hi, T], None, 0, T, T)[0], dtype=I32))
        if spoil:
            for t in (c.q, c.k, c.v, c.do):
                t[lo:hi:3, ::5] = bad
        runs.append(c.run(B).got())
    for name, t in runs[1].items():
        same = torch.equal if name != "lse" else lambda x, y: torch.equal(x, y)
        axis = 2 if name == "lse" else 1
        for part in (slice(0, lo), slice(hi, T)):
            x, y = [r[name].transpose(1, axis)[:, part] for r in runs]
            assert same(x, y), name
    assert bool(runs[1]["o"][0, lo].isnan().all())      # and where they are seen, they show


def test_keys_that_nothing_sees_may_hold_anything(B):
    for kind, shape in (("ragged", (3, 1, 700, 16, 2, 128)), ("any", (2, 40, 300, 4, 2, 64))):
        c = Case(kind, *shape)
        sp = c.span.clamp(0, shape[2]).long()
        j = torch.arange(shape[2], device=DEV)
        unseen = ~((j >= sp[..., :1]) & (j < sp[..., 1:])).any(1)
        assert bool(unseen.any())
        for t in (c.k, c.v):
            t[:shape[0] * shape[2]][unseen.reshape(-1)] = NAN
        c.run(B).check()


def test_rows_that_lie_on_one_key(B):
    """Scores so sharp that nearly all weight is on one key: dP - delta cancels, and a delta that carried o's rounding would show in dq and dk."""
    for d in (64, 128):
        c = Case("causal", 1, 260, 260, 8, 2, d, std=16.0).run(B)
        c.check()
        want = c.want()
        for name, limit in (("dq", 6e-3), ("dk", 6e-3), ("dv", 4e-3), ("o", 4e-3)):      # one to three roundings of 2^-8, spread evenly: 1.7e-3 each
            x = c.got()[name].double()
            assert float((x - want[name][0]).norm() / want[name][0].norm()) < limit, name


def test_the_same_bits_every_time_and_on_another_stream(B):
    for shape in (("docs", 1, 517, 517, 8, 2, 128), ("ragged", 3, 1, 700, 16, 2, 128)):
        first = {k: t.clone() for k, t in Case(*shape, cap=20.0).run(B).got().items()}
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        again = Case(*shape, cap=20.0)
        torch.cuda.synchronize()
        again.run(B, stream=side.cuda_stream)
        for name, t in again.got().items():
            assert torch.equal(t, first[name]), name
