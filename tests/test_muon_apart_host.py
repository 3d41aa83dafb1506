"""Tensors that stand for two matrices of a call, told by their addresses, without a GPU."""
import pytest

from paper_2509_04084_amd import lowdiff as ld


@pytest.mark.parametrize("written,read", [([], []), ([1, 2], []), ([1, 2], [3, 3]), ([], [1, 1])])
def test_apart(written, read):
    ld._apart("outs", written, read)


@pytest.mark.parametrize("written,read", [([1, 1], []), ([1, 2], [3, 2]), ([1, 2, 1], [4]), ([5], [5])])
def test_not_apart(written, read):
    with pytest.raises(ValueError, match="outs: a tensor stands for two matrices"):
        ld._apart("outs", written, read)
