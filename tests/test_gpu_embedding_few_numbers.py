"""The embedding's gradient for tables of one to three rows and many tokens: digits of one or two bits, and scratch whose parts still lie on 16-byte boundaries."""
import pytest

import pack_reference as R
from test_gpu_embedding import B, DEV, stream, tokens  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("kind", ["one", "even", "zipf"])
@pytest.mark.parametrize("T,V,h", [(8193, 1, 8), (9000, 1, 264), (20001, 1, 40), (9000, 2, 40), (9000, 3, 72), (129, 1, 40)])
def test_gradient(B, T, V, h, kind, accumulate):  # noqa: F811
    g = torch.Generator().manual_seed(T + V)
    ids = tokens(kind, T, V, g).to(DEV)
    dx = torch.randn((T, h), generator=g).to(torch.bfloat16).to(DEV)
    given = torch.randn((V, h), generator=g).to(DEV)
    dt = given.clone()
    n = B.rp_op_embed_scratch(T, V, h)
    ws = torch.full((n // 4 + 64,), float("nan"), device=DEV)
    B.rp_op_embed_bwd(stream(), dx, h, ids, 0.5, dt, h, accumulate, T, V, h, ws[:n // 4])
    want, bound = R.embedding_gradient(dx, ids, 0.5, V, given if accumulate else None)
    assert bool(((dt.double() - want).abs() <= bound + 1e-30).all())
    assert bool(ws[n // 4:].isnan().all())


def test_a_table_without_rows(B):  # noqa: F811
    """No row, no table: every token is padding."""
    ids = torch.arange(-2, 5, dtype=torch.int32, device=DEV)
    x = torch.full((8, 40), float("nan"), dtype=torch.bfloat16, device=DEV)
    B.rp_op_embed_fwd(stream(), None, 40, ids, 2.0, x, 40, 7, 0, 40)
    assert bool((x[:7] == 0).all()) and bool(x[7].isnan().all())
    B.rp_op_embed_bwd(stream(), x, 40, ids, 2.0, None, 40, 0, 7, 0, 40, None)      # (nothing to write)
