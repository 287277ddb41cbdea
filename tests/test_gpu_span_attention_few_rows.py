"""Few rows: o together with what its rounding left over.

Each weight goes to the product in two bf16 parts, off by 2^-8 of 2^-8 of it at most; scores are fp32 sums of up to 128 products (2^-24 of the sum of their absolute values, a root of 128 of them by chance:
1e-6 of scores of up to 10), exponentials are off by 2^-22, and o's second part by 2^-16 of o.  All of that is below 6e-5 of a row's spread, and less in a norm, where it adds up by chance.  A weight in one
part, off by 2^-9 and more by chance, would show as 5e-4 or more."""
import pytest

from test_gpu_span_attention import B, Case  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("kind,b,nq,nk,a,kh,d,scratch", [("ragged", 3, 1, 700, 16, 2, 128, "full"), ("all", 2, 1, 4096, 8, 8, 128, "full"), ("all", 1, 3, 2000, 8, 2, 64, "full"), ("all", 1, 8, 500, 8, 2, 128, "least"),
                                                         ("any", 1, 1, 3000, 4, 2, 64, "least")])
def test_o_and_its_rest(B, kind, b, nq, nk, a, kh, d, scratch, cap):  # noqa: F811
    c = Case(kind, b, nq, nk, a, kh, d, cap=cap, std=1.0).run(B, scratch, backward=False).check(backward=False)
    want = c.want()["o"][0]
    got = c.view(c.o, nq).double() + c.view(c.rest, nq).double()
    assert float((got - want).norm() / want.norm()) < 1e-4
