"""What the binding takes as an address: a tensor, a number or None.  Bytes and text are host memory that ctypes would pass on as if it were the device's."""
import pytest

import __graft_entry__
from paper_2604_27085_amd import build as _build
import os
if not os.path.exists(_build.LIB):
    __graft_entry__.build()
from paper_2604_27085_amd import binding as B  # noqa: E402

np = pytest.importorskip("numpy")
torch = pytest.importorskip("torch")


def test_tensors_numbers_and_none():
    t = torch.zeros(3)
    assert B._ptr(t) == t.data_ptr() and B._ptr(4096) == 4096 and B._ptr(None) is None


@pytest.mark.parametrize("what", [b"bytes", "text", bytearray(8), 1.5, np.zeros(3), [1, 2]])
def test_anything_else_is_refused(what):
    with pytest.raises(AttributeError):
        B._ptr(what)
    with pytest.raises(AttributeError):
        B.rp_op_rmsnorm_fwd(None, what, None, None, None, 0, 8, 1e-6)
