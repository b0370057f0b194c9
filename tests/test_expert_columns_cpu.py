"""eqb_quant_cols by entries needs the length of the lists: without it every entry would
be taken for a token's number."""
import pytest
import torch

import paper_2609_28053_gb300 as eqb


def test_entries_without_their_lists_length_are_refused():
    x = torch.zeros(4, 16, dtype=torch.bfloat16)
    off = torch.zeros(3, dtype=torch.int32)
    entry = torch.zeros(8, dtype=torch.int32)
    with pytest.raises(ValueError, match="needs K"):
        eqb.eqb_quant_cols(x, off, off, entry)
    with pytest.raises(ValueError, match="needs K"):
        eqb.eqb_quant_cols(x, off, off, entry=entry, err_flag=None)
    with pytest.raises(ValueError, match="CUDA"):  # the next check's turn
        eqb.eqb_quant_cols(x, off, off, entry, 2)
    with pytest.raises(ValueError, match="CUDA"):
        eqb.eqb_quant_cols(x, off, off)
