"""What the reading calls refuse before they touch a GPU, beside the list in test_reading_oracle (no GPU needed)."""
import ctypes

import pytest

from paper_2604_18913_amd import reading
from test_reading_oracle import _attention, _status


@pytest.mark.parametrize("name", ["q_row", "k_row", "v_row"])
@pytest.mark.parametrize("stride", [-8, -128, -(1 << 40), 1 << 23])
def test_row_strides_outside_their_range(name, stride):
    # (the gradients' loads take a row's size as an unsigned number)
    a = _attention(**{name: stride})
    rc, text = _status("logoskg_attend", a)
    assert rc == 1 and "row stride" in text
    grad = reading._AttentionGrad(struct_size=64, dout=64, dq=64, dk=64, dv=64, workspace=64, workspace_bytes=1 << 20)
    rc, text = _status("logoskg_attend_backward", a, grad)
    assert rc == 1 and "row stride" in text
    assert reading._load().logoskg_attend_backward_bytes(ctypes.addressof(a)) == -1
