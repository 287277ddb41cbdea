"""Embedding and its gradient, dropout, the plan of packed rows."""
import pytest

import pack_reference as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
NAN = float("nan")


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_27085_amd import binding
    return binding


def stream():
    return torch.cuda.current_stream().cuda_stream


def tokens(kind, T, V, g):
    if kind == "one":
        return torch.full((T,), V - 1, dtype=I32)
    if kind == "even":
        return torch.randint(0, V, (T,), generator=g, dtype=I32)
    if kind == "none":
        return torch.full((T,), -100, dtype=I32)
    ids = torch.exp(torch.rand(T, generator=g) * torch.log(torch.tensor(float(V)))).long().sub(1).clamp(0, V - 1).to(I32)
    ids[torch.rand(T, generator=g) < 0.2] = -1      # padding
    ids[torch.rand(T, generator=g) < 0.05] = V      # and numbers that are too large
    return ids


@pytest.mark.parametrize("T,V,h,pad,scale", [(1, 1, 8, 0, 1.0), (8, 50, 4096, 0, 1.0), (300, 1000, 264, 8, 16.25), (1023, 7, 2056, 0, 1.0), (5000, 151936, 64, 0, 8.0)])
def test_rows(B, T, V, h, pad, scale):
    g = torch.Generator().manual_seed(T)
    ids = tokens("zipf", T, V, g).to(DEV)
    table = torch.full((V, h + pad), NAN, dtype=BF16)
    table[:, :h] = torch.randn((V, h), generator=g).to(BF16)
    table = table.to(DEV)
    x = torch.full((T + 1, h + 2 * pad), NAN, dtype=BF16, device=DEV)
    B.rp_op_embed_fwd(stream(), table, h + pad, ids, scale, x, h + 2 * pad, T, V, h)
    at = (ids >= 0) & (ids < V)
    want = torch.where(at[:, None], (table[ids.clamp(0, V - 1).long(), :h].float() * scale).to(BF16), 0.0)      # the one rounding of an exact product
    assert torch.equal(x[:T, :h], want)
    assert bool(x[T:].isnan().all()) and bool(x[:, h:].isnan().all())


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("kind", ["zipf", "one", "even", "none"])
@pytest.mark.parametrize("T,V,h", [(1, 1, 8), (7, 1000, 264), (32, 40, 64), (1000, 33, 2056), (1024, 5000, 40), (1025, 5000, 40), (3001, 1024, 136), (8192, 151936, 40), (9000, 151936, 64), (9000, 900, 40),
                                   (70000, 3000, 8)])
def test_gradient(B, T, V, h, kind, accumulate):
    g = torch.Generator().manual_seed(T + V)
    ids = tokens(kind, T, V, g).to(DEV)
    dx = torch.randn((T, h), generator=g).to(BF16).to(DEV)
    given = torch.randn((V, h), generator=g).to(DEV) if accumulate else None
    n = B.rp_op_embed_scratch(T, V, h)
    runs = []
    for _ in range(2):
        ws = torch.full((n // 4 + 4,), NAN, device=DEV)
        dt = given.clone() if accumulate else torch.full((V, h), NAN, device=DEV)
        B.rp_op_embed_bwd(stream(), dx, h, ids, 2.5, dt, h, accumulate, T, V, h, ws[:n // 4])
        torch.cuda.synchronize()
        assert bool(ws[n // 4:].isnan().all())
        runs.append(dt)
    assert torch.equal(*runs)      # the same bits every time
    want, bound = R.embedding_gradient(dx, ids, 2.5, V, given)
    off = (runs[0].double() - want).abs() / (bound + 1e-36)
    assert float(off.max()) <= 1.0
    if accumulate:                 # other rows are left alone
        at = torch.ones(V, dtype=torch.bool, device=DEV)
        at[ids[(ids >= 0) & (ids < V)].long()] = False
        assert torch.equal(runs[0][at], given[at])


@pytest.mark.parametrize("kind", ["zipf", "one", "even"])
@pytest.mark.parametrize("T", [63, 64, 65, 127, 128, 129, 2047, 2048, 4097, 8191, 8193])
def test_gradient_around_the_sorts_limits(B, T, kind):
    test_gradient(B, T, 700, 72, kind, 0)


def test_gradient_strides_and_nothing_to_do(B):
    T, V, h = 50, 20, 40
    g = torch.Generator().manual_seed(3)
    ids = tokens("zipf", T, V, g).to(DEV)
    dx = torch.full((T, h + 8), NAN, dtype=BF16, device=DEV)
    dx[:, :h] = torch.randn((T, h), generator=g).to(BF16).to(DEV)
    dt = torch.full((V + 1, h + 16), NAN, device=DEV)
    ws = torch.empty(B.rp_op_embed_scratch(T, V, h), dtype=torch.uint8, device=DEV)
    B.rp_op_embed_bwd(stream(), dx, h + 8, ids, 1.0, dt, h + 16, 0, T, V, h, ws)
    want, bound = R.embedding_gradient(dx[:, :h], ids, 1.0, V)
    assert bool(((dt[:V, :h].double() - want).abs() <= bound).all())
    assert bool(dt[V:].isnan().all()) and bool(dt[:, h:].isnan().all())
    B.rp_op_embed_bwd(stream(), None, h, None, 1.0, dt, h + 16, 0, 0, V, h, ws)      # no tokens: the gradient is zero
    assert bool((dt[:V, :h] == 0).all())
    dt.fill_(3.0)
    B.rp_op_embed_bwd(stream(), None, h, None, 1.0, dt, h + 16, 1, 0, V, h, None)
    assert bool((dt == 3.0).all())
    B.rp_op_embed_fwd(stream(), dt, h, None, 1.0, None, h, 0, V, h)


def test_the_same_row_for_two_tokens_against_differences(B):
    """The sum of <x, w> moves with a row of the table by scale times the sum of w over its tokens: dx = w is that derivative, exactly linear."""
    T, V, h = 40, 9, 16
    g = torch.Generator().manual_seed(9)
    ids = torch.randint(0, V, (T,), generator=g, dtype=I32).to(DEV)
    w = torch.randint(-8, 9, (T, h), generator=g).to(BF16).to(DEV)
    dt = torch.empty((V, h), device=DEV)
    B.rp_op_embed_bwd(stream(), w, h, ids, 0.5, dt, h, 0, T, V, h, torch.empty(B.rp_op_embed_scratch(T, V, h), dtype=torch.uint8, device=DEV))
    x = torch.empty((2, T, h), dtype=BF16, device=DEV)
    for v in range(V):
        for e in (0, 7, 15):
            for s in (0, 1):      # values that bf16 and the sums hold exactly
                table = torch.zeros((V, h), dtype=BF16, device=DEV)
                table[v, e] = (-2.0, 2.0)[s]
                B.rp_op_embed_fwd(stream(), table, h, ids, 0.5, x[s], h, T, V, h)
            d = ((x[1].double() - x[0].double()) * w.double()).sum() / 4.0
            assert float(d) == float(dt[v, e])


# ---------------------------------------------------------------------------------------------------- dropout
@pytest.mark.parametrize("res", [False, True])
@pytest.mark.parametrize("T,n,p,pad", [(1, 8, 0.5, 0), (3, 40, 0.1, 0), (17, 264, 0.9, 8), (5, 2056, 0.0, 0), (5, 64, 1.0, 8), (300, 8, 0.3, 16)])
def test_dropout(B, T, n, p, pad, res):
    g = torch.Generator().manual_seed(T + n)
    seed, offset = 0x123456789ABCDEF1, (1 << 63) + 77
    x = torch.full((T + 1, n + pad), NAN, dtype=BF16)
    x[:T, :n] = torch.randn((T, n), generator=g).to(BF16)
    r = torch.randn((T, n + 2 * pad), generator=g).to(BF16)
    x, r = x.to(DEV), r.to(DEV)
    y = torch.full((T + 1, n + 8), NAN, dtype=BF16, device=DEV)
    step = torch.tensor([5], dtype=torch.int64, device=DEV)
    B.rp_op_dropout(stream(), x, n + pad, r if res else None, n + 2 * pad, y, n + 8, T, n, p, seed, offset, step)
    stay, share = R.stays(T, n, p, seed, offset + 5)
    stay = stay.to(DEV)
    want = torch.where(stay, x[:T, :n].double() / max(share, 1e-9), 0.0)
    size = want.abs()
    if res:
        want, size = want + r[:, :n].double(), size + r[:, :n].double().abs()
    got = y[:T, :n].double()
    assert bool(((got - want).abs() <= R.H * want.abs() + 2.0 ** -22 * size).all())
    assert bool(y[T:].isnan().all()) and bool(y[:, n:].isnan().all())
    # in place, and the backward call: the same mask
    if pad == 0:
        z = x[:T].clone()
        B.rp_op_dropout(stream(), z, n, r if res else None, n, z, n, T, n, p, seed, offset + 5)
        assert torch.equal(z, y[:T, :n])


def test_dropout_of_infinities_and_of_a_large_array(B):
    """What is dropped may be infinite; and the share that stays, in groups whose number passes 2^20."""
    x = torch.full((4096, 4096), float("inf"), dtype=BF16, device=DEV)
    y = torch.empty_like(x)
    B.rp_op_dropout(stream(), x, 4096, None, 0, y, 4096, 4096, 4096, 0.25, 11, 3)
    assert bool(((y == 0) | torch.isinf(y)).all())
    kept = float(torch.isinf(y).double().mean())
    assert abs(kept - 0.75) < 5 * (0.25 * 0.75 / y.numel()) ** 0.5      # five standard deviations
    stay, _ = R.stays(1, 4096, 0.25, 11, 3)
    assert torch.equal(torch.isinf(y[:1]).cpu(), stay)
    rows = torch.isinf(y).double()
    both = float((rows[:, :-1] * rows[:, 1:]).mean())                   # neighbours do not know of one another
    assert abs(both - 0.75 ** 2) < 1e-3


# ---------------------------------------------------------------------------------------------------- the plan
@pytest.mark.parametrize("starts,prefix,window,T,seq", [
    ([0, 10, 10, 37, 60], None, 0, 64, 64), ([3, 9, 30], [2, 50], 0, 40, 20), ([0, 5, 100], [3, 7], 4, 90, 30), ([0, 300], [17], 0, 300, 300), ([0], None, 0, 7, 7),
    ([5, 5, 5], [1, 1], 2, 10, 5)])
def test_plan(B, starts, prefix, window, T, seq):
    dev = lambda v: torch.tensor(v, dtype=I32, device=DEV)  # noqa: E731
    span, pos, first = torch.full((T + 1, 2), -7, dtype=I32, device=DEV), dev([-7] * (T + 1)), torch.full((T + 1,), 9, dtype=torch.uint8, device=DEV)
    B.rp_op_pack_plan(stream(), dev(starts), dev(prefix) if prefix else None, len(starts) - 1, window, T, seq, span, pos, first)
    want = R.plan(starts, prefix, window, T, seq)
    assert span.tolist() == [list(v) for v in want[0]] + [[-7, -7]]
    assert pos.tolist() == want[1] + [-7] and first.tolist() == want[2] + [9]
    B.rp_op_pack_plan(stream(), dev(starts), None, len(starts) - 1, 0, T, seq, None, pos, None)
    assert pos.tolist() == want[1] + [-7]
    B.rp_op_pack_plan(stream(), None, None, 0, 0, 0, 1)
