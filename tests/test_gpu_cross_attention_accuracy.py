"""Cross attention's gradients of ordinary and of sharp rows, with the key loop in one piece and in slices, inside limits that the stored output's delta or a
dS in one bf16 part would leave (attention_accuracy, test_cross_attention_limits)."""
import math

import pytest

import attention_accuracy as A

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_27085_amd import binding
    return binding


def gradients(B, q, k, v, do, sliced):
    """One sequence: q, do [m, a, d]; k, v [n, kh, d]; with `sliced`, as much scratch as the calls make use of."""
    (m, a, d), (n, kh, _) = q.shape, k.shape
    st = torch.cuda.current_stream().cuda_stream
    q, k, v, do = [t.to(DEV) for t in (q, k, v, do)]
    fwd, bwd = B.rp_op_cross_attn_scratch(1, m, n, a, kh, d)
    assert bwd or not sliced
    ws = torch.full((max(fwd, bwd) // 4,), float("nan"), device=DEV) if sliced else None
    nan = lambda t: torch.full_like(t, float("nan"))  # noqa: E731
    o, dq, dk, dv = nan(q), nan(q), nan(k), nan(v)
    lse = torch.full((1, a, m), float("nan"), device=DEV)
    delta = nan(lse)
    qd, kd, lens = a * d, kh * d, (None, None, 1, m, n, a, kh, d, d ** -0.5, ws)
    B.rp_op_cross_attn_fwd(st, q, k, v, o, lse, qd, kd, kd, qd, *lens)
    B.rp_op_cross_attn_bwd(st, q, k, v, o, do, lse, delta, dq, dk, dv, qd, kd, kd, qd, qd, qd, kd, kd, *lens)
    torch.cuda.synchronize()
    return {"dq": dq.cpu(), "dk": dk.cpu()}


def inputs(m, n, a, kh, d, gain=None, std=2.0):
    g = torch.Generator().manual_seed(m + n + d)
    k, v, do = [torch.randn(s, generator=g).to(torch.bfloat16) for s in ((n, kh, d), (n, kh, d), (m, a, d))]
    q = A.sharp_queries(k.float(), a, m, gain, g) if gain else std * torch.randn((m, a, d), generator=g)
    return q.to(torch.bfloat16), k, v, do


def check(got, want, limits):
    for name, limit in limits:
        value, bound = want[name]
        off, worst = A.distance(got[name], value), float(((got[name].double() - value).abs() / bound).nan_to_num(nan=math.inf).max())
        assert off < limit and worst <= 1.0, (name, off, worst)


EXACT_DELTA = 256      # keys up to which delta comes from the scores
# keys; whether the loop over them is cut into slices (eleven tiles and more, with scratch)
LOOPS = [(129, False), (256, False), (257, False), (700, False), (700, True), (1500, False), (1500, True), (5000, True)]


@pytest.mark.parametrize("n,sliced,std", [x + (1.0,) for x in LOOPS] + [x + (2.0,) for x in LOOPS if x[0] <= EXACT_DELTA or x[1]])
@pytest.mark.parametrize("d", [64, 128])
def test_ordinary_rows(B, d, n, sliced, std):
    x = inputs(200, n, 4, 2, d, std=std)
    check(gradients(B, *x, sliced), A.gradients(*x, d ** -0.5, sliced or n <= EXACT_DELTA), [("dq", A.DQ_ORDINARY)])


@pytest.mark.parametrize("n,sliced", LOOPS + [(300, False), (705, False)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("share", [1.0, 3.0])
def test_keys_that_share_a_part(B, share, d, n, sliced):
    """A part that all keys have in common (a bias) adds the same to every score of a row and nothing to dq, since a row of dS sums up to zero; what delta is off by
    times it would show.  Against the mean of 64 keys 1 / 64 of the centred keys' square is left besides sum P^2: sqrt(2) u sqrt(0.03 + 1 / 64) = 0.3 u
    beside dq's own rounding u, 1.74e-3."""
    q, k, v, do = inputs(200, n, 4, 2, d, std=1.0)
    k = (k.float() + share * torch.randn((1, 2, d), generator=torch.Generator().manual_seed(n))).to(torch.bfloat16)
    x = (q, k, v, do)
    check(gradients(B, *x, sliced), A.gradients(*x, d ** -0.5, sliced or n <= EXACT_DELTA), [("dq", A.DQ_ORDINARY)])


@pytest.mark.parametrize("n,sliced", LOOPS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gain", [1.0, 1.2])
def test_sharp_rows(B, gain, d, n, sliced):
    """Rows that put nearly all of their weight on one key, where dP - delta cancels."""
    x = inputs(200, n, 4, 2, d, gain * math.sqrt(128.0 / d))
    exact = sliced or n <= EXACT_DELTA
    check(gradients(B, *x, sliced), A.gradients(*x, d ** -0.5, exact), [("dq", A.DQ_SHARP_EXACT if exact else A.DQ_SHARP), ("dk", A.DK_SHARP)])


@pytest.mark.parametrize("scratch", ["none", "full"])
@pytest.mark.parametrize("d", [64, 128])
def test_sharp_rows_of_a_padded_batch(B, d, scratch):
    """Sequences of different lengths, as columns of larger arrays, whose unused rows hold NaN: each row's own place, query and delta."""
    from test_gpu_cross_attention import Case
    c = Case(3, 200, 700, 6, 2, d, [200, 77, 5], [700, 300, 257], pad=8)
    b, nq, nk, a, kh, _ = c.shape
    g = torch.Generator().manual_seed(d)
    q, k, v, do = [c.view(t, n) for t, n in ((c.q, nq), (c.k, nk), (c.v, nk), (c.do, nq))]
    for i in range(b):
        q[i, :c.ql[i]] = A.sharp_queries(k[i, :c.kl[i]].float().cpu(), a, c.ql[i], 1.1 * math.sqrt(128.0 / d), g).to(DEV)
    c.run(B, scratch)
    got = c.got()
    for i in range(b):
        m, n = c.ql[i], c.kl[i]
        want = A.gradients(*[t.cpu() for t in (q[i, :m], k[i, :n], v[i, :n], do[i, :m])], c.scale, False)
        check({"dq": got["dq"][i, :m].cpu(), "dk": got["dk"][i, :n].cpu()}, want, [("dq", A.DQ_SHARP), ("dk", A.DK_SHARP)])
        assert float(got["dq"][i, m:].abs().sum()) == 0.0 and float(got["dk"][i, n:].abs().sum()) == 0.0
