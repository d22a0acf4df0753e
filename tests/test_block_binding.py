"""What the binding of include/symb_block.h makes of the strides that torch's tensors have.  No GPU is touched."""
import pytest
import torch

from paper_2507_03220_amd import binding as sb


def _rows(T, heads, dim, apart):
    return torch.zeros(max(T, 1) * apart, dtype=torch.bfloat16).as_strided((T, heads, dim), (apart, dim, 1))


@pytest.mark.parametrize("apart", [128, 132, 200, 1001])
def test_the_stride_of_a_single_row_says_nothing(apart):
    """One row lies nowhere apart from another: a decode step's tensor is as good as any, whatever it is cut from (the C entry takes multiples of 8)."""
    one = _rows(1, 2, 64, apart)
    assert one.stride(0) == apart and sb._head_rows(one, "q", (1, 2, 64)) == 128
    assert sb._head_rows(torch.zeros(2, 64, 1, dtype=torch.bfloat16).permute(2, 0, 1), "q", (1, 2, 64)) == 128
    assert sb._head_rows(_rows(0, 2, 64, apart), "q", (0, 2, 64)) == 128


def test_the_stride_of_several_rows_is_theirs():
    assert sb._head_rows(_rows(3, 2, 64, 200), "q", (3, 2, 64)) == 200
    with pytest.raises(ValueError):
        sb._head_rows(_rows(3, 2, 64, 200).transpose(0, 1).contiguous().transpose(0, 1), "q", (3, 2, 64))
