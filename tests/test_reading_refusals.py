"""What the reading calls refuse and ask for before they touch a GPU, beside the list in test_reading_oracle (no GPU needed)."""
import ctypes

import pytest
import torch

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


@pytest.mark.parametrize("docs, rows, keys, ordered", [(100_000, 30, 70, False), (1024, 18, 78, False), (8, 500, 500, True), (1024, 120, 300, True), (7, 500, 500, False)])
def test_blocks_are_ordered_where_documents_are_many_and_long(docs, rows, keys, ordered):
    # the room for the order is what tells: a block is 128 rows or keys, and each document has one more than it fills
    a = _attention(num_docs=docs, num_rows=docs * rows, num_keys=docs * keys, heads=32, kv_heads=32, q_row=2048, k_row=2048, v_row=2048)
    blocks = (docs * rows >> 7) + (docs * keys >> 7) + 2 * docs
    assert reading._load().logoskg_attend_backward_bytes(ctypes.addressof(a)) == docs * rows * 32 * 4 + (blocks * 4 if ordered else 0)


def test_a_bias_without_buckets_is_refused():
    # (its tensor has no memory, and no place is what the library takes for no bias)
    with pytest.raises(ValueError, match="a bucket at least"):
        reading._score(None, 0.0, torch.zeros(2, 0), torch.zeros(9, dtype=torch.int32), 2, 64, torch.float32, -1)
    assert reading._score(None, 0.0, torch.zeros(2, 1), torch.zeros(9, dtype=torch.int32), 2, 64, torch.float32, -1)[4:] == (1, 4)
