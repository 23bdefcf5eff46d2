"""A 4-bit matrix keeps the tensors and sizes that were checked when it was made."""
import pytest

from paper_1905_05233_amd import sequence_ops as S


@pytest.mark.parametrize("name", ["tiles", "scales", "rows", "cols", "group", "other"])
def test_attributes_cannot_be_set(name):
    w = S.W4Matrix.__new__(S.W4Matrix)
    with pytest.raises(AttributeError):
        setattr(w, name, 1)
