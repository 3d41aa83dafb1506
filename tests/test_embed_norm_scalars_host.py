"""Tensors without a dimension where the embedding's entry points take rows: refused as other shapes are."""
import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld


@pytest.mark.parametrize("place", ["table", "pos_table", "out", "dout", "grad"])
def test_a_tensor_without_dimensions_is_refused(place):
    ids, one, row = torch.zeros(1, dtype=torch.int64), torch.tensor(1.0), torch.ones(1, 1)
    at = {name: one if name == place else row for name in ("table", "pos_table", "out", "dout", "grad")}
    with pytest.raises((TypeError, ValueError)):
        if place in ("dout", "grad"):
            ld.ld_embed_grad(at["dout"], ids, at["grad"])
        else:
            ld.ld_embed_lookup(at["table"], ids, 1.0, at["pos_table"], ids, out=at["out"])
