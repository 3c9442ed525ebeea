"""What the binding of the paged cache makes of index tensors, without a GPU."""
import pytest
import torch

from paper_2405_12532_b200 import binding as pb


class _Host(pb.PyrPages):
    """The checks alone: no handle, tensors on the host."""

    def __init__(self):
        self._index, self.device = -1, torch.device("cpu")


@pytest.mark.parametrize("n,groups,rows", [(3, 4, 0), (1, 4, 0), (3, 1, 0), (0, 4, 5), (3, 4, 1), (3, 1, 7), (1, 4, 7), (3, 4, 7)])
def test_index_lists_of_any_number_of_rows_are_taken(n, groups, rows):
    """None at all among them (torch gives dimensions without elements strides as if they had one)."""
    p = _Host()
    idx = torch.zeros(n, groups, rows, dtype=torch.int32)
    ptr, g, stride = p._idx(idx, n)
    assert (ptr, g) == (idx.data_ptr(), groups) and stride == (idx.stride(0) if n > 1 else 0)
    p.handle = None


@pytest.mark.parametrize("idx", [torch.zeros(3, 7, 4, dtype=torch.int32).transpose(1, 2), torch.zeros(3, 4, 14, dtype=torch.int32)[:, :, ::2],
                                 torch.zeros(3, 4, 9, dtype=torch.int32)[:, :, :7], torch.zeros(3, 4, 7), torch.zeros(3, 28, dtype=torch.int32),
                                 torch.zeros(2, 4, 7, dtype=torch.int32)])
def test_index_lists_that_are_not_contiguous_are_refused(idx):
    with pytest.raises(ValueError):
        _Host()._idx(idx, 3)
