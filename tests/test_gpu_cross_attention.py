"""Cross attention, forward and backward, against 64-bit attention with bounds counted from its bf16 roundings (ops_reference)."""
import pytest

import ops_reference as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
BF16 = torch.bfloat16
EXACT_DELTA = 128      # keys up to which the backward takes delta from the scores


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_27085_amd import binding
    return binding


def stream():
    return torch.cuda.current_stream().cuda_stream


class Case:
    """Inputs and outputs inside larger arrays: `pad` columns beside the heads and `guard` rows behind the last sequence, all of them NaN, as
    is what the lengths leave unused of the inputs."""

    def __init__(self, b, nq, nk, a, kh, d, q_len=None, kv_len=None, pad=0, seed=0, std=2.0):
        self.shape = (b, nq, nk, a, kh, d)
        g = torch.Generator().manual_seed(seed + 7 * nq + 11 * nk + a + d)
        self.ql, self.kl = q_len or [nq] * b, kv_len or [nk] * b
        self.q_len = torch.tensor(q_len, dtype=torch.int32, device=DEV) if q_len else None
        self.kv_len = torch.tensor(kv_len, dtype=torch.int32, device=DEV) if kv_len else None
        self.pad = pad

        def array(n, heads, lens, std):
            t = torch.full((b * n + 2, heads * d + 2 * pad), float("nan"), dtype=BF16)
            if std:
                for i in range(b):
                    t[i * n:i * n + lens[i], pad:pad + heads * d] = (std * torch.randn((lens[i], heads * d), generator=g)).to(BF16)
            return t.to(DEV)

        self.q, self.do = array(nq, a, self.ql, std), array(nq, a, self.ql, 1.0)
        self.k, self.v = array(nk, kh, self.kl, 1.0), array(nk, kh, self.kl, 1.0)
        self.o, self.dq = array(nq, a, None, 0), array(nq, a, None, 0)
        self.dk, self.dv = array(nk, kh, None, 0), array(nk, kh, None, 0)
        nan = lambda: torch.full((b * a * nq + 16,), float("nan"), device=DEV)  # noqa: E731
        self.lse, self.delta = nan(), nan()
        self.scale = d ** -0.5

    def view(self, t, n):
        b, _, _, _, _, d = self.shape
        return t[:b * n, self.pad:t.shape[1] - self.pad].reshape(b, n, (t.shape[1] - 2 * self.pad) // d, d)

    def run(self, B, scratch="full", backward=True, lse=True):
        b, nq, nk, a, kh, d = self.shape
        fwd, bwd = B.rp_op_cross_attn_scratch(b, nq, nk, a, kh, d)
        size = {"full": max(fwd, bwd), "none": 0, "some": max(fwd, bwd) // 2}[scratch] if isinstance(scratch, str) else scratch
        ws = torch.full((size // 4,), float("nan"), device=DEV) if size else None
        at = lambda t: t.data_ptr() + 2 * self.pad  # noqa: E731
        ld = lambda t: t.shape[1]  # noqa: E731
        B.rp_op_cross_attn_fwd(stream(), at(self.q), at(self.k), at(self.v), at(self.o), self.lse if lse else None, ld(self.q), ld(self.k), ld(self.v), ld(self.o),
                               self.q_len, self.kv_len, b, nq, nk, a, kh, d, self.scale, ws)
        if backward:
            B.rp_op_cross_attn_bwd(stream(), at(self.q), at(self.k), at(self.v), at(self.o), at(self.do), self.lse, self.delta, at(self.dq), at(self.dk), at(self.dv),
                                   ld(self.q), ld(self.k), ld(self.v), ld(self.o), ld(self.do), ld(self.dq), ld(self.dk), ld(self.dv), self.q_len, self.kv_len,
                                   b, nq, nk, a, kh, d, self.scale, ws)
        torch.cuda.synchronize()
        return self

    def got(self):
        b, nq, nk, a, kh, d = self.shape
        return {"o": self.view(self.o, nq), "lse": self.lse[:b * a * nq].reshape(b, a, nq), "dq": self.view(self.dq, nq), "dk": self.view(self.dk, nk),
                "dv": self.view(self.dv, nk)}

    def check(self, backward=True):
        b, nq, nk, a, kh, d = self.shape
        want = R.cross_attention(self.view(self.q, nq), self.view(self.k, nk), self.view(self.v, nk), self.view(self.do, nq), self.ql, self.kl, self.scale,
                                 lambda n: n <= EXACT_DELTA)
        got = self.got()
        for name in ("o", "lse", "dq", "dk", "dv") if backward else ("o", "lse"):
            x, (y, bound) = got[name].double(), want[name]
            same = (x == y)      # infinities
            off = torch.where(same, 0.0, (x - y).abs())
            worst = float((off / (bound + 1e-30)).nan_to_num(nan=float("inf")).max()) if x.numel() else 0.0
            assert bool((off <= bound + 1e-30).all()), (name, worst)
        # columns beside the heads and rows behind the last sequence
        for t, n in ((self.o, nq), (self.dq, nq), (self.dk, nk), (self.dv, nk)) if backward else ((self.o, nq),):
            assert bool(torch.isnan(t[b * n:]).all())
            if self.pad:
                assert bool(torch.isnan(t[:, :self.pad]).all() and torch.isnan(t[:, -self.pad:]).all())
        assert bool(torch.isnan(self.lse[b * a * nq:]).all())
        if backward:
            assert bool(torch.isnan(self.delta[b * a * nq:]).all())


SHAPES = [
    # b, nq, nk, a, kh, d, q_len, kv_len
    (1, 1, 1, 1, 1, 64, None, None), (1, 1, 1, 8, 1, 128, None, None), (2, 1, 64, 16, 2, 128, None, None), (3, 5, 65, 6, 2, 64, None, None),
    (1, 2, 3, 4, 2, 128, None, None), (2, 127, 129, 4, 4, 128, None, None), (2, 33, 300, 8, 2, 64, [33, 12], [300, 0]),
    (3, 70, 140, 4, 2, 128, [1, 70, 0], [140, 77, 64]), (4, 64, 128, 2, 1, 64, [64, 63, 1, 0], [0, 128, 1, 127]), (1, 200, 1000, 4, 1, 128, None, None),
    (8, 1, 1500, 16, 8, 128, None, [1500, 3, 0, 700, 64, 65, 1, 1499]), (1, 1, 9000, 8, 8, 128, None, None), (2, 3, 5000, 32, 4, 64, [3, 2], [5000, 129]),
    (1, 640, 640, 8, 8, 128, None, None), (1, 4000, 100, 8, 2, 128, None, None), (2, 1500, 70, 8, 2, 64, [1500, 611], [70, 5]), (1, 513, 31, 16, 16, 64, None, None),
    (5, 17, 515, 4, 2, 128, [17, 1, 16, 9, 0], [515, 512, 513, 0, 200]), (1, 31, 513, 5, 5, 64, None, None), (2, 16, 2048, 64, 4, 128, None, [2048, 1025]),
    # one workgroup of eight waves a key head
    (3, 2, 300, 32, 2, 128, [2, 1, 2], [300, 0, 131]), (2, 1, 300, 16, 16, 64, None, [257, 300]), (2, 5, 290, 12, 2, 64, [5, 4], [290, 33]),
]


@pytest.mark.parametrize("b,nq,nk,a,kh,d,q_len,kv_len", SHAPES)
def test_against_the_formulas(B, b, nq, nk, a, kh, d, q_len, kv_len):
    Case(b, nq, nk, a, kh, d, q_len, kv_len).run(B).check()


@pytest.mark.parametrize("b,nq,nk,a,kh,d,q_len,kv_len", [SHAPES[3], SHAPES[7], SHAPES[10], SHAPES[15]])
def test_columns_of_larger_arrays(B, b, nq, nk, a, kh, d, q_len, kv_len):
    Case(b, nq, nk, a, kh, d, q_len, kv_len, pad=24).run(B).check()


@pytest.mark.parametrize("scratch", ["none", "some"])
@pytest.mark.parametrize("b,nq,nk,a,kh,d,q_len,kv_len", [SHAPES[10], SHAPES[11], SHAPES[12], SHAPES[14], SHAPES[19]])
def test_less_scratch(B, b, nq, nk, a, kh, d, q_len, kv_len, scratch):
    Case(b, nq, nk, a, kh, d, q_len, kv_len).run(B, scratch).check()


@pytest.mark.parametrize("d,nk", [(128, 130), (64, 70)])
def test_many_rows(B, d, nk):
    """1024 workgroups of 256 rows and more: the eight-wave kernels at d = 128."""
    Case(4, 2048, nk, 32, 8, d, [2048, 2047, 2048, 1000], [nk, nk, 1, nk]).run(B).check()


def test_one_array_for_keys_and_values(B):
    """k | v, and dk | dv, as the columns of one array each, as a fused projection leaves and takes them."""
    b, nq, nk, a, kh, d = 2, 40, 90, 8, 2, 64
    c = Case(b, nq, nk, a, kh, d, None, [90, 33])
    kv = torch.cat((c.k, c.v), 1)
    dkv = torch.full_like(kv, float("nan"))
    st, w = stream(), kh * d
    B.rp_op_cross_attn_fwd(st, c.q, kv, kv[:, w:], c.o, c.lse, a * d, 2 * w, 2 * w, a * d, None, c.kv_len, b, nq, nk, a, kh, d, c.scale)
    B.rp_op_cross_attn_bwd(st, c.q, kv, kv[:, w:], c.o, c.do, c.lse, c.delta, c.dq, dkv, dkv[:, w:], a * d, 2 * w, 2 * w, a * d, a * d, a * d, 2 * w, 2 * w, None,
                           c.kv_len, b, nq, nk, a, kh, d, c.scale)
    torch.cuda.synchronize()
    c.dk, c.dv = dkv[:, :w].contiguous(), dkv[:, w:].contiguous()
    c.check()


def test_lse_is_optional_and_runs_repeat(B):
    """Without lse the same output; twice the same bits (nothing is added in an order that timing decides)."""
    for shape in (SHAPES[10], SHAPES[12], SHAPES[14], SHAPES[7]):
        x, y, z = Case(*shape).run(B), Case(*shape).run(B), Case(*shape).run(B, backward=False, lse=False)
        for name, t in x.got().items():
            assert torch.equal(t, y.got()[name]), name
        assert torch.equal(x.got()["o"], z.got()["o"])
        assert bool(torch.isnan(z.lse).all())


def test_sharp_rows(B):
    """Scores of some hundred: one key takes the whole weight; the running maximum moves late (keys in ascending order of their score)."""
    c = Case(1, 64, 700, 4, 2, 128, std=20.0)
    k = c.k[:700].float()
    order = (k[:, :128] @ c.q[0, :128].float()).argsort()
    c.k[:700] = c.k[:700][order]
    c.run(B).check()


def test_a_length_out_of_range_counts_as_the_nearest(B):
    x = Case(2, 20, 70, 4, 2, 64, [20, 0], [0, 70])
    x.q_len = torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32, device=DEV)
    x.kv_len = torch.tensor([-1, 71], dtype=torch.int32, device=DEV)
    x.run(B).check()


def test_empty_lengths(B):
    """No queries: dk and dv are zero.  No keys: o and dq are zero, lse -inf.  No sequences: nothing."""
    x = Case(2, 0, 70, 4, 2, 64)
    x.run(B).check()
    y = Case(2, 20, 0, 4, 2, 128)
    y.run(B).check()
    Case(0, 20, 30, 4, 2, 128).run(B)


def test_two_calls_at_once(B):
    """Two streams, each with its own scratch."""
    cases = [Case(*SHAPES[12], seed=s) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, s in zip(cases, streams):
            b, nq, nk, a, kh, d = c.shape
            if not hasattr(c, "ws"):
                c.ws = torch.empty(max(B.rp_op_cross_attn_scratch(b, nq, nk, a, kh, d)), dtype=torch.uint8, device=DEV)
                torch.cuda.synchronize()
            qd, kd = a * d, kh * d
            B.rp_op_cross_attn_fwd(s.cuda_stream, c.q, c.k, c.v, c.o, c.lse, qd, kd, kd, qd, c.q_len, c.kv_len, b, nq, nk, a, kh, d, c.scale, c.ws)
            B.rp_op_cross_attn_bwd(s.cuda_stream, c.q, c.k, c.v, c.o, c.do, c.lse, c.delta, c.dq, c.dk, c.dv, qd, kd, kd, qd, qd, qd, kd, kd, c.q_len, c.kv_len, b, nq,
                                   nk, a, kh, d, c.scale, c.ws)
    torch.cuda.synchronize()
    for c in cases:
        c.check()


def test_a_sequence_past_two_to_the_32_bytes(B):
    """Keys whose rows lie 16 KB apart over 5 GB: the far ones are read, and their gradients written, where they are."""
    b, nq, nk, a, kh, d, ld = 1, 2, 330000, 2, 1, 64, 8192
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 25 GB")
    c = Case(b, nq, nk, a, kh, d)
    wide = lambda t: torch.empty((nk, ld), dtype=BF16, device=DEV)  # noqa: E731
    K, V, dK, dV = wide(0), wide(0), wide(0), wide(0)
    K[:, :d], V[:, :d] = c.k[:nk], c.v[:nk]
    ws = torch.empty(max(B.rp_op_cross_attn_scratch(b, nq, nk, a, kh, d)), dtype=torch.uint8, device=DEV)
    B.rp_op_cross_attn_fwd(stream(), c.q, K, V, c.o, c.lse, a * d, ld, ld, a * d, None, None, b, nq, nk, a, kh, d, c.scale, ws)
    B.rp_op_cross_attn_bwd(stream(), c.q, K, V, c.o, c.do, c.lse, c.delta, c.dq, dK, dV, a * d, ld, ld, a * d, a * d, a * d, ld, ld, None, None, b, nq, nk, a, kh, d,
                           c.scale, ws)
    torch.cuda.synchronize()
    c.dk[:nk], c.dv[:nk] = dK[:, :d], dV[:, :d]
    c.check()
