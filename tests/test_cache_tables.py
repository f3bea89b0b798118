"""Block tables whose rows overlap are refused before anything is launched (no GPU needed: the check comes before that of the device)."""
import pytest
import torch

from paper_2511_22972_b200 import cache


def make(table, sequences):
    p = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16)
    return cache.PagedCache(p, p.clone(), table, torch.zeros(sequences, dtype=torch.int32))


@pytest.mark.parametrize("table", [
    torch.zeros(1, 4, dtype=torch.int32).expand(3, -1),              # one row for all
    torch.zeros(32, dtype=torch.int32).as_strided((3, 4), (2, 1)),
    torch.zeros(32, dtype=torch.int32).as_strided((3, 4), (3, 1)),
    torch.zeros(1, 1, dtype=torch.int32).expand(3, 1),
])
def test_tables_whose_rows_overlap_are_refused(table):
    with pytest.raises(ValueError, match="overlap"):
        make(table, 3)


@pytest.mark.parametrize("table", [
    torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, 9, dtype=torch.int32)[:, :4], torch.zeros(1, 4, dtype=torch.int32),
    torch.zeros(9, dtype=torch.int32).as_strided((1, 4), (0, 1)), torch.zeros(3, 9, dtype=torch.int32)[:, :1],
])
def test_other_tables_go_on_to_the_next_check(table):
    with pytest.raises(ValueError, match="CUDA device"):
        make(table, len(table))
