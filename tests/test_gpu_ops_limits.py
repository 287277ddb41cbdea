"""Calls of the layer operators that need more than one launch, since a launch has fewer than 2^32 threads."""
import pytest

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


def test_a_rotation_of_more_than_two_to_the_32_threads(B):
    """2^24 + 5 tokens with 255 units each, in place.  They repeat every 4096, and so do their positions, so every block of 4096 has to be what a call of
    4096 tokens gives, bit for bit."""
    T, n, d, rot, seq = (1 << 24) + 5, 4096, 512, 510, 8
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    g = torch.Generator(device=DEV).manual_seed(1)
    few = torch.empty((n, d), dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    cs = torch.empty((seq, rot // 2, 2), device=DEV).normal_(generator=g)
    x = torch.empty((T, d), dtype=torch.bfloat16, device=DEV)
    whole = T // n * n
    x[:whole].view(-1, n, d).copy_(few.expand(whole // n, n, d))
    x[whole:] = few[:T - whole]
    turn = lambda t: B.rp_op_rope(stream(), 0, 0, d, rot, t, None, d, 0, t, None, d, 0, cs, seq, None, t.shape[0], seq, 1, 0)  # noqa: E731
    before = few.clone()
    turn(few)
    turn(x)
    torch.cuda.synchronize()
    assert not torch.equal(few, before)
    for part in x[:whole].view(-1, n, d).split(256):
        assert bool((part.view(torch.int16) == few.view(torch.int16)).all())
    assert torch.equal(x[whole:], few[:T - whole])


@pytest.mark.parametrize("masked", [False, True])
def test_a_balance_loss_of_more_than_two_to_the_22_groups(B, masked):
    """A group a token: what is chosen has all of the group's weight, f = 1 / top_k on it."""
    from test_gpu_balance import check, run
    T, E, k = (1 << 22) + 3, 8, 2
    g = torch.Generator(device=DEV).manual_seed(2)
    x = 2.0 * torch.randn((T, E), generator=g, device=DEV)
    idx = x.topk(k, 1).indices.to(torch.int32)
    mask = (torch.rand(T, generator=g, device=DEV) < 0.7).to(torch.uint8) if masked else None
    keep = mask.bool() if masked else torch.ones(T, dtype=torch.bool, device=DEV)
    counts = torch.zeros((T, E), dtype=torch.float64, device=DEV).scatter_(1, idx.long(), 1.0) * keep[:, None]
    f, p, N = counts / k, x.double().softmax(1) * keep[:, None], int(keep.sum())
    dot, lse = (f * p).sum(1, keepdim=True), torch.where(keep, torch.logsumexp(x.double(), 1), 0.0)
    bal, z = E / N * dot.sum(), lse.square().sum() / N
    part = lambda sign: 0.5 * p * (0.2 * E / N * (f + sign * dot) + 0.1 * 2 / N * (lse if sign < 0 else lse.abs())[:, None])  # noqa: E731
    want = (counts.long(), torch.cat((keep, keep.sum()[None])), torch.stack((0.2 * bal + 0.1 * z, bal, z)), part(-1), part(1))
    check(run(B, x, idx, mask, 1, k, 0.2, 0.1, 0.5), want)
