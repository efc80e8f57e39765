"""What an output of the rotation may look like, without a device: the kernel fills a token's heads side by side, so a view whose
rows are anything else would have its gaps, or memory behind its last element, written."""
import pytest
import torch

import paper_2511_07423_b200 as syn
from paper_2511_07423_b200 import binding

T, H, HD = 3, 4, 64


def take(y, heads=H, tokens=T):
    x = torch.zeros(tokens, heads, HD)
    return binding._heads("q", x, y, None, tokens, HD, torch.float32, -1)


@pytest.mark.parametrize("make", [
    lambda: torch.zeros(T, 2 * H, HD)[:, :, :HD // 2],                                      # twice the heads, half as wide
    lambda: torch.zeros(1000).as_strided((T, H // 2, 2 * HD), (300, HD, 1)),                # wide heads that overlap
    lambda: torch.zeros(1000).as_strided((T, 1, H * HD), (300, HD, 1)),                     # one head of all
    lambda: torch.zeros(T, H, HD + 8)[:, :, :HD],                                           # heads apart
    lambda: torch.zeros(H, T, HD).transpose(0, 1),                                          # head by head
    lambda: torch.zeros(T, H, 2 * HD)[:, :, ::2],                                           # every other component
    lambda: torch.zeros(T, H * HD + 8)[:, :H * HD],                                         # (rows apart: in three dimensions only)
])
def test_outputs_that_are_not_a_tokens_heads_side_by_side_are_refused(make):
    y = make()
    assert y.numel() == T * H * HD and not y.is_contiguous()
    with pytest.raises(syn.SynError) as e:
        take(y)
    assert e.value.code == -1


@pytest.mark.parametrize("shape", [(T, H, HD), (T, H * HD), (1, T, H, HD), (T * H * HD,)])
def test_contiguous_outputs_of_any_shape_are_taken(shape):
    y = torch.zeros(shape)
    h = take(y)
    assert (h.y, h.y_stride, h.n_heads) == (y.data_ptr(), H * HD, H)


def test_slices_of_rows_are_taken():
    y = torch.zeros(T, H + 2, HD)[:, 1:H + 1]
    assert (take(y).y, take(y).y_stride) == (y.data_ptr(), (H + 2) * HD)
    one = torch.zeros(T, 5, 2 * HD)[:, 2:3, :HD]              # one head: the distance to the next does not matter
    assert (take(one, 1).y, take(one, 1).y_stride) == (one.data_ptr(), 10 * HD)
    row = torch.zeros(1, 9, HD)[:, :H]                          # one token: nor that to the next
    assert take(row, tokens=1).y_stride == H * HD
