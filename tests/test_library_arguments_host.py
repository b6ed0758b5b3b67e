"""What the binding takes for an address: tensors, arrays, whole numbers and None, nothing else."""
import numpy as np
import pytest

from paper_2009_14783_amd import binding as hs


@pytest.mark.parametrize("bad", [b"abcd", "abcd", [1, 2], 1.0])
def test_other_objects_are_no_address(bad):
    with pytest.raises(AttributeError):      # an empty product: a call that takes the operand is fine
        hs.hs_op_gemm_fp8(0, 5, 7, bad, 128, None, 4, None, 128, None, 4, None, 5, stream=0)


def test_addresses():
    torch = pytest.importorskip("torch")
    a, t = np.zeros(4), torch.zeros(4)
    assert hs._ptr(a) == a.ctypes.data and hs._ptr(t) == t.data_ptr() and hs._ptr(4096) == 4096 and hs._ptr(None) is None
