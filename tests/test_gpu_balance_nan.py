"""A valid token whose logits are all NaN: the losses say so, as its gradient does; a padded one's NaN stays out, and a row of -inf adds nothing."""
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


@pytest.mark.parametrize("T,seq,E,k", [(64, 64, 1, 1), (64, 64, 16, 2), (60, 20, 129, 3), (5000, 5000, 64, 2), (300, 300, 1024, 8)])
@pytest.mark.parametrize("how", ["all", "all and -inf", "one"])
def test_nan_shows_in_every_loss(B, T, seq, E, k, how):
    from test_gpu_balance import make, run
    logits, idx, _, _ = make(T, seq, E, k)
    row = 7
    if how == "all":
        logits[row] = float("nan")
    else:
        if how == "all and -inf":
            logits[row] = -float("inf")
        logits[row, E // 2] = float("nan")
    counts, tokens, loss, d = run(B, logits, idx, None, seq, k, 0.3, 0.02, 1.0)
    assert bool(torch.isnan(loss).all()) and bool(torch.isnan(d[row]).all())
    others = torch.arange(T, device=DEV) != row
    assert bool(torch.isfinite(d[others]).all()) and int(tokens[-1]) == T
    mask = others.to(torch.uint8)
    logits[3] = -float("inf")
    _, tokens, loss, d = run(B, logits, idx, mask, seq, k, 0.3, 0.02, 1.0)
    assert bool(torch.isfinite(loss).all() and torch.isfinite(d).all()) and int(tokens[-1]) == T - 1
    assert float(d[row].abs().max()) == 0.0 and float(d[3].abs().max()) == 0.0
