"""The router's balance loss, its counts and its gradient against the 64-bit formulas."""
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


def make(T, seq, E, k, masked=False, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + T + E)
    logits = 2.0 * torch.randn((T, E), generator=g, device=DEV) + torch.randn(E, generator=g, device=DEV)
    idx = logits.topk(k, 1).indices.to(torch.int32)
    mask = (torch.rand(T, generator=g, device=DEV) < 0.7).to(torch.uint8) if masked else None
    given = 1e-3 * torch.randn((T, E), generator=g, device=DEV)
    return logits, idx, mask, given


def run(B, logits, idx, mask, seq, k, coef, z, gs, given=None, grad=True, in_place=False, shift=0):
    T, E = logits.shape
    G = T // seq
    counts = torch.full((G * E + 8,), -7, dtype=torch.int32, device=DEV)
    tokens = torch.full((G + 9,), -7, dtype=torch.int32, device=DEV)
    loss = torch.full((8,), float("nan"), device=DEV)
    out = torch.full((T * E + 8 + shift,), float("nan"), device=DEV)
    d = out[shift:shift + T * E].view(T, E)
    if in_place:
        d.copy_(given)
    ws = torch.full((B.rp_op_moe_balance_scratch(T, seq, E),), 255, dtype=torch.uint8, device=DEV)
    B.rp_op_moe_balance(stream(), logits, idx, mask, T, seq, E, k, coef, z, gs, counts, tokens, loss, d if in_place else given, d if grad else None, ws)
    torch.cuda.synchronize()
    assert bool((counts[G * E:] == -7).all() and (tokens[G + 1:] == -7).all() and torch.isnan(loss[3:]).all() and torch.isnan(out[shift + T * E:]).all())
    if not grad:
        assert bool(torch.isnan(out).all())
    return counts[:G * E].view(G, E), tokens[:G + 1], loss[:3], d


def check(got, want, given=None, grad=True):
    """fp32 arithmetic: an exponential of an argument of some tens is off by 1e-6 to 4e-6, sums and products of the row by less; 1e-5 of the
    terms in all.  The sum with what was there rounds once more."""
    counts, tokens, loss, d = got
    wc, wt, wl, wg, terms = want
    assert torch.equal(counts.long(), wc) and torch.equal(tokens.long(), wt.to(tokens.device))
    assert bool(((loss.double() - wl).abs() <= 1e-5 * wl.abs() + 1e-30).all()), (loss, wl)
    if grad:
        base = given.double() if given is not None else 0.0
        bound = 1e-5 * terms + 2.0 ** -23 * (base + wg).abs() + 1e-30
        assert bool(((d.double() - base - wg).abs() <= bound).all())


SIZES = [(1, 1, 1, 1), (1, 1, 8, 2), (3, 3, 2, 1), (37, 37, 7, 3), (256, 256, 32, 4), (300, 100, 60, 8), (64, 16, 16, 16), (1000, 1000, 128, 8), (999, 333, 129, 2),
         (515, 515, 256, 8), (260, 130, 257, 1), (130, 130, 512, 8), (99, 33, 1000, 6), (70, 7, 1023, 4), (64, 64, 1024, 64), (5000, 5000, 64, 2), (40000, 40000, 8, 2)]


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("T,seq,E,k", SIZES)
def test_against_the_formulas(B, T, seq, E, k, masked):
    logits, idx, mask, given = make(T, seq, E, k, masked)
    want = R.balance(logits, idx, mask, seq, k, 0.3, 0.02, -1.5)
    check(run(B, logits, idx, mask, seq, k, 0.3, 0.02, -1.5), want)
    check(run(B, logits, idx, mask, seq, k, 0.3, 0.02, -1.5, given), want, given)


def test_gradient_in_place_left_out_and_off_16_byte_boundaries(B):
    T, seq, E, k = 120, 40, 32, 4
    logits, idx, mask, given = make(T, seq, E, k, True)
    want = R.balance(logits, idx, mask, seq, k, 1.0, 0.1, 2.0)
    check(run(B, logits, idx, mask, seq, k, 1.0, 0.1, 2.0, given, in_place=True), want, given)
    check(run(B, logits, idx, mask, seq, k, 1.0, 0.1, 2.0, grad=False), want, grad=False)
    check(run(B, logits, idx, mask, seq, k, 1.0, 0.1, 2.0, given, shift=1), want, given)
    x = torch.empty(T * E + 1, device=DEV)[1:].view(T, E)
    x.copy_(logits)
    check(run(B, x, idx, mask, seq, k, 1.0, 0.1, 2.0), want)


@pytest.mark.parametrize("T,seq,masked", [(3000, 1, True), (3000, 1, False), (70000, 1, True), (2100, 3, True)])
def test_many_groups(B, T, seq, masked):
    logits, idx, mask, given = make(T, seq, 8, 2, masked)
    x, i = logits, idx
    # the loop over groups of the 64-bit form, all groups at once
    E, k = 8, 2
    keep = mask.bool() if masked else torch.ones(T, dtype=torch.bool, device=DEV)
    one = torch.zeros((T, E), dtype=torch.float64, device=DEV).scatter_add_(1, i.long(), torch.ones((T, k), dtype=torch.float64, device=DEV)) * keep[:, None]
    counts = one.reshape(-1, seq, E).sum(1)
    n = keep.reshape(-1, seq).sum(1)
    f = (counts / (n.clamp(min=1)[:, None] * k)).repeat_interleave(seq, 0)
    p = x.double().softmax(1) * keep[:, None]
    N = int(n.sum())
    dot = (f * p).sum(1, keepdim=True)
    lse = torch.where(keep, torch.logsumexp(x.double(), 1), 0.0)
    bal, z = E / N * dot.sum(), lse.square().sum() / N
    grad = 0.5 * p * (0.2 * E / N * (f - dot) + 0.1 * 2 / N * lse[:, None])
    terms = 0.5 * p * (0.2 * E / N * (f + dot) + 0.1 * 2 / N * lse.abs()[:, None])
    want = (counts.long(), torch.cat((n, n.sum()[None])), torch.stack((0.2 * bal + 0.1 * z, bal, z)), grad, terms)
    check(run(B, x, i, mask, seq, k, 0.2, 0.1, 0.5), want)


def test_rows_without_probabilities_and_numbers_that_are_no_expert(B):
    """A row of -inf alone; experts that are closed to a token; padding that holds NaN; choices out of range or twice the same."""
    T, seq, E, k = 96, 48, 16, 3
    logits, idx, _, given = make(T, seq, E, k)
    mask = torch.ones(T, dtype=torch.uint8, device=DEV)
    mask[40:48], mask[90:] = 0, 0
    logits[40:48] = float("nan")
    logits[91, 3] = float("inf")
    logits[5] = -float("inf")
    logits[7, :15] = -float("inf")
    logits[50:60, 4:9] = torch.finfo(torch.float32).min
    idx[3, 0], idx[4, 1], idx[6, 2], idx[60, 0] = -1, 16, 2 ** 31 - 1, -2 ** 31
    idx[10, :] = 5
    clean = torch.where(mask.bool()[:, None], logits, 0.0)
    want = R.balance(clean, idx, mask, seq, k, 0.5, 0.01, 1.0)
    check(run(B, logits, idx, mask, seq, k, 0.5, 0.01, 1.0, given), want, given)


def test_no_valid_token_and_no_token(B):
    logits, idx, _, given = make(64, 32, 8, 2)
    mask = torch.zeros(64, dtype=torch.uint8, device=DEV)
    counts, tokens, loss, d = run(B, logits, idx, mask, 32, 2, 1.0, 1.0, 1.0, given)
    assert int(counts.abs().sum()) == 0 and int(tokens.abs().sum()) == 0 and float(loss.abs().sum()) == 0 and torch.equal(d, given)
    tokens, loss = torch.full((1,), 3, dtype=torch.int32, device=DEV), torch.ones(3, device=DEV)
    B.rp_op_moe_balance(stream(), None, None, None, 0, 4, 8, 2, 1.0, 1.0, 1.0, None, tokens, loss, None, None, None)
    torch.cuda.synchronize()
    assert int(tokens) == 0 and float(loss.abs().sum()) == 0


def test_gradient_against_differences_of_the_loss(B):
    """(loss(x + h u) - loss(x - h u)) / 2h with the kernel's own fp32 loss: off by its rounding, 2^-22 of the loss over h, and h^2 of the third
    derivative (below 1e-3 of the first at h = 0.02 on these inputs' scale)."""
    T, E, k = 64, 16, 2
    logits, idx, _, _ = make(T, T, E, k)
    u = torch.randn((T, E), device=DEV, generator=torch.Generator(device=DEV).manual_seed(3))
    h = 0.02
    at = lambda s: float(run(B, logits + s * u, idx, None, T, k, 1.0, 0.1, 1.0)[2][0].double())  # noqa: E731
    _, _, loss, d = run(B, logits, idx, None, T, k, 1.0, 0.1, 1.0)
    want = float((d.double() * u).sum())
    # third derivatives of a softmax average are below 6 |u|^3 of its terms; E / N sum_t bounds them by their mean
    third = 6 * float(u.abs().amax(1).pow(3).mean()) * (float(loss[1]) + 0.1 * (2 * float(loss[2]) ** 0.5 + 6)) * h * h / 6
    assert abs((at(h) - at(-h)) / (2 * h) - want) <= third + 2.0 ** -21 * float(loss[0]) / h


def test_runs_repeat(B):
    logits, idx, mask, given = make(4004, 1001, 256, 8, True)
    x = run(B, logits, idx, mask, 1001, 8, 0.01, 1e-3, 0.5, given)
    y = run(B, logits, idx, mask, 1001, 8, 0.01, 1e-3, 0.5, given)
    for s, t in zip(x, y):
        assert torch.equal(s, t)
