"""What evict_to_pages refuses before anything is launched (no GPU needed): lengths that the selection's kernel could not write."""
import pytest
import torch

from paper_2510_07651_b200 import api


def _args(lens, H=4, table_lists=(2, 4)):
    k = torch.zeros((96, 1, 16, 128), dtype=torch.bfloat16)
    q, rows = torch.zeros((2, 8, 16, 128), dtype=torch.bfloat16), torch.zeros((2, H, 300, 128), dtype=torch.bfloat16)
    return q, rows, rows, api.PagedCache(k, k, torch.zeros(table_lists + (12,), dtype=torch.int32), lens)


@pytest.mark.parametrize("lens", [torch.zeros((1, 4), dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32), torch.zeros((2, 4), dtype=torch.int64),
                                  torch.zeros((2, 4), dtype=torch.int16), torch.zeros((2, 4), dtype=torch.int32, device="meta")])
def test_lengths_of_another_shape_type_or_device(lens):
    with pytest.raises(ValueError, match="the selection writes"):
        api.evict_to_pages(*_args(lens), budget=40, safeguard=0.2)


def test_before_the_score():
    with pytest.raises(ValueError, match="list per head"):
        api.evict_to_pages(*_args(torch.zeros((2,), dtype=torch.int32)), budget=40, safeguard=0.2)
    with pytest.raises(ValueError, match="share memory"):
        api.evict_to_pages(*_args(torch.zeros((1,), dtype=torch.int32).expand(2), table_lists=(2,)), budget=40)
    with pytest.raises(ValueError, match="budget"):
        api.evict_to_pages(*_args(torch.zeros((2,), dtype=torch.int32)), budget=400)
    with pytest.raises(ValueError, match="CUDA tensor"):
        api.evict_to_pages(*_args(torch.zeros((2, 4), dtype=torch.int32)), budget=40, safeguard=0.2)
