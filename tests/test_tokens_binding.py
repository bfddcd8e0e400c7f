"""Refusals of the binding's calls on packed tokens: an error of the library, whatever is wrong with a tensor.  No GPU."""
import pytest
import torch

from paper_2406_10774_amd import binding
from test_tokens_abi import Caller


@pytest.mark.parametrize("kw", [dict(tree_mask=torch.zeros(6, dtype=torch.int64)), dict(tree_mask=torch.zeros(6, 1, 1, dtype=torch.int64)),
                                dict(topk_idx=torch.zeros(2, 40, dtype=torch.int32)), dict(topk_idx=torch.zeros(80, dtype=torch.int32)),
                                dict(topk_idx=torch.zeros(2, 8, 5, 1, dtype=torch.int32)),
                                dict(topk_idx=torch.zeros(2, 16, 5, dtype=torch.int32))])       # a list a query head, of 16
def test_masks_and_lists_of_other_shapes(kw):
    with pytest.raises(binding.QuestError, match="have to be"):
        Caller().tree(**kw)
