"""The plan of packed rows, key by key: who sees whom where documents, rows, a window and prefixes meet."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
I32 = torch.int32


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_27085_amd import binding
    return binding


def sees(t, j, starts, prefix, window, seq):
    """Whether token t sees token j."""
    doc = next((i for i in range(len(starts) - 1) if starts[i] <= t < starts[i + 1]), None)
    if doc is None or not starts[doc] <= j < starts[doc + 1] or t // seq != j // seq:
        return False
    if window and j <= t - window:      # before the last `window` up to itself, also within a prefix
        return False
    end = starts[doc] + (prefix[doc] if prefix else 0)
    return j <= t or (t < end and j < end)


@pytest.mark.parametrize("window", [0, 1, 3, 16, 1000])
@pytest.mark.parametrize("starts,prefix,T,seq", [([0, 64], [20], 64, 64), ([2, 11, 11, 40, 59], [5, 3, 17, 100], 64, 64), ([0, 25, 70], [9, 30], 90, 30), ([0, 25, 70], None, 90, 30), ([0, 10, 20], [0, -4], 24, 24)])
def test_who_sees_whom(B, starts, prefix, T, seq, window):
    dev = lambda v: torch.tensor(v, dtype=I32, device=DEV)  # noqa: E731
    span = torch.full((T, 2), -7, dtype=I32, device=DEV)
    B.rp_op_pack_plan(torch.cuda.current_stream().cuda_stream, dev(starts), dev(prefix) if prefix else None, len(starts) - 1, window, T, seq, span, None, None)
    for t, (lo, hi) in enumerate(span.tolist()):
        row = t // seq * seq
        want = [j for j in range(T) if sees(t, j, starts, prefix, window, seq)]
        assert list(range(row + lo, row + hi)) == want, t
