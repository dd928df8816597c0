"""What the mixture-of-experts bindings refuse before they reach the library, on CPU tensors and stand-ins."""
import pytest
import torch

from paper_2405_01943_b200 import binding as b

CPU = torch.device("cpu")


def test_rows_used_is_the_last_of_the_offsets():
    """The address of the number of rows in use: never one outside the tensor."""
    offsets = torch.zeros(5, dtype=torch.int32)
    assert b._rows_used(offsets, CPU) == offsets.data_ptr() + 16
    assert b._rows_used(offsets[:1], CPU) == offsets.data_ptr()
    assert b._rows_used(None, CPU) is None
    for bad in (offsets[:0], offsets.long(), offsets[::2], offsets.view(1, 5)):
        with pytest.raises(ValueError):
            b._rows_used(bad, CPU)
