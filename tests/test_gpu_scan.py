"""The gated linear recurrence, forward and backward, against 64 bits (pack_reference)."""
import pytest

import pack_reference as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
NAN = float("nan")


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_27085_amd import binding
    return binding


class Case:
    def __init__(self, weight, b, n, c, docs=False, length=None, state=True, pad=0, seed=0, shift=3.0):
        self.dims, self.weight, self.pad, self.length = (b, n, c), weight, pad, length
        g = torch.Generator().manual_seed(seed + n + c)

        def array(std, shift=0.0):
            t = torch.full((b * n + 2, c + 2 * pad), NAN, dtype=BF16)
            if std:
                t[:b * n, pad:pad + c] = (std * torch.randn((b * n, c), generator=g) + shift * torch.rand(c, generator=g)).to(BF16)
            return t.to(DEV)

        self.x, self.g, self.dy = array(1.0), array(2.0, shift), array(1.0)
        self.y, self.dx, self.dg = array(0), array(0), array(0)
        if length:
            for i, m in enumerate(length):
                for t in (self.x, self.g, self.dy):
                    t[i * n + m:(i + 1) * n] = NAN      # what is behind a length may hold anything
        self.len = torch.tensor(length, dtype=torch.int32, device=DEV) if length else None
        self.first = (torch.rand((b, n), generator=g) < 0.02).to(torch.uint8).mul(3).to(DEV) if docs else None
        self.h0 = torch.randn((b, c), generator=g).to(DEV) if state else None
        self.dlast = torch.randn((b, c), generator=g).to(DEV) if state else None
        full = lambda: torch.full((b * c + 8,), NAN, device=DEV)  # noqa: E731
        self.last, self.dh0 = full(), full()

    def run(self, B, backward=True, stream=None):
        b, n, c = self.dims
        st = stream or torch.cuda.current_stream().cuda_stream
        states, scratch = B.rp_op_scan_sizes(b, n, c)
        self.states = torch.full((states // 4 + 8,), NAN, device=DEV) if backward else None
        ws = torch.full((scratch // 4,), NAN, device=DEV) if scratch else None
        at = lambda t: t.data_ptr() + 2 * self.pad  # noqa: E731
        ld = c + 2 * self.pad
        B.rp_op_scan_fwd(st, self.weight, at(self.x), at(self.g), at(self.y), ld, ld, ld, self.first, self.len, self.h0, self.last, self.states, b, n, c, ws)
        if backward:
            B.rp_op_scan_bwd(st, self.weight, at(self.x), at(self.g), at(self.dy), at(self.dx), at(self.dg), ld, ld, ld, ld, ld, self.first, self.len, self.states,
                             self.dlast, self.dh0, b, n, c, ws)
        torch.cuda.synchronize()
        if backward:
            assert bool(self.states[states // 4:].isnan().all())
        return self

    def view(self, t):
        b, n, c = self.dims
        return t[:b * n, self.pad:self.pad + c].reshape(b, n, c)

    def got(self):
        b, n, c = self.dims
        return {"y": self.view(self.y), "last": self.last[:b * c].reshape(b, c), "dx": self.view(self.dx), "dg": self.view(self.dg), "dh0": self.dh0[:b * c].reshape(b, c)}

    def check(self, names=("y", "last", "dx", "dg", "dh0")):
        b, n, c = self.dims
        on = torch.stack([torch.arange(n, device=DEV) < m for m in (self.length or [n] * b)])[..., None] if b else torch.zeros((0, n, 1), dtype=torch.bool, device=DEV)
        clean = [torch.where(on, self.view(t), 0.0) for t in (self.x, self.g, self.dy)]
        want = R.scan(self.weight, *clean, self.first, self.length, self.h0, self.dlast)
        for name in names:
            value, bound = want[name]
            x = self.got()[name].double()
            assert bool(torch.isfinite(x).all()), name
            off = (x - value).abs() / (bound + 1e-36)
            assert not off.numel() or float(off.max()) <= 1.0, (name, float(off.max()))
        for t in (self.y, self.dx, self.dg):
            inside = torch.zeros_like(t, dtype=torch.bool)
            inside[:b * n, self.pad:self.pad + c] = True
            assert bool(t[~inside].isnan().all())
        assert bool(self.last[b * c:].isnan().all()) and bool(self.dh0[b * c:].isnan().all())
        return self


@pytest.mark.parametrize("weight", [0, 1, 2])
@pytest.mark.parametrize("b,n,c", [(1, 1, 8), (2, 1, 264), (1, 7, 64), (3, 64, 256), (2, 65, 520), (1, 200, 1024), (4, 333, 72), (1, 1500, 40), (2, 4096, 16)])
def test_forward_and_backward(B, weight, b, n, c):
    Case(weight, b, n, c).run(B).check()


@pytest.mark.parametrize("b,n,c,docs", [(3, 1200, 2304, True), (1, 1153, 7304, False), (2, 4500, 136, True), (1, 9001, 8, False)])
def test_many_chunks(B, b, n, c, docs):
    """More chunks a sequence than are looked at at once, with workgroups for more than one round, and with few."""
    Case(2, b, n, c, docs=docs).run(B).check()


@pytest.mark.parametrize("weight", [0, 1, 2])
def test_documents_lengths_and_strides(B, weight):
    Case(weight, 2, 500, 136, docs=True, state=False).run(B).check()
    Case(weight, 3, 300, 72, docs=True, length=[300, 0, 129]).run(B).check()
    Case(weight, 5, 70, 40, length=[64, 63, 65, 1, 70], pad=8).run(B).check()
    Case(weight, 2, 20, 40, docs=True, length=[1, 0], pad=16).run(B).check()


@pytest.mark.parametrize("shift", [-40.0, 12.0, 60.0])
def test_gates_near_zero_and_one(B, shift):
    for weight in (0, 1, 2):
        Case(weight, 1, 700, 64, shift=shift).run(B).check()


def test_without_tokens_the_state_is_passed_on(B):
    c = Case(1, 2, 0, 40).run(B)
    assert torch.equal(c.got()["last"], c.h0) and torch.equal(c.got()["dh0"], c.dlast)
    Case(1, 0, 9, 40).run(B)


def test_step_by_step_is_the_whole(B):
    """The step of a generation, state in place: the numbers of one call over all tokens.  That one composes the maps of eight tokens before it
    applies them, so the two differ by roundings of fp32; where those lie on either side of a border of bf16, y differs by one step, 2^-7 of the value at most."""
    whole = Case(2, 2, 50, 264).run(B, backward=False)
    b, n, c = whole.dims
    st = torch.cuda.current_stream().cuda_stream
    h = whole.h0.clone()
    x, g = whole.view(whole.x), whole.view(whole.g)
    y = torch.empty((b, 1, c), dtype=BF16, device=DEV)
    for t in range(n):
        B.rp_op_scan_fwd(st, 2, x[:, t].contiguous(), g[:, t].contiguous(), y, c, c, c, None, None, h, h, None, b, 1, c)
        want = whole.view(whole.y)[:, t].double()
        assert bool(((y[:, 0].double() - want).abs() <= 2.0 ** -7 * want.abs() + 1e-5).all()), t
    last = whole.got()["last"]
    assert float((h - last).abs().max()) <= 1e-5 * float(last.abs().max())


def test_a_document_does_not_reach_the_next(B):
    for n in (40, 900):
        runs = []
        for bad in (None, NAN, float("inf")):
            c = Case(1, 1, n, 64, state=True)
            c.first = torch.zeros((1, n), dtype=torch.uint8, device=DEV)
            c.first[0, n // 2] = 1
            if bad is not None:
                c.x[:n // 2, ::3] = bad
                c.dy[n // 2:n, 1::3] = bad
            runs.append(c.run(B).got())
        for r in runs[1:]:
            assert torch.equal(r["y"][:, n // 2:], runs[0]["y"][:, n // 2:]) and torch.equal(r["last"], runs[0]["last"])
            assert torch.equal(r["dx"][:, :n // 2], runs[0]["dx"][:, :n // 2]) and torch.equal(r["dh0"], runs[0]["dh0"])


def test_in_place_and_another_stream(B):
    c = Case(1, 2, 300, 136, docs=True)
    want = {k: t.clone() for k, t in Case(1, 2, 300, 136, docs=True).run(B).got().items()}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    c.dx, c.dg = c.dy, c.g      # the gradients take their inputs' places
    c.run(B, stream=side.cuda_stream)
    for name, t in c.got().items():
        assert torch.equal(t, want[name]), name
