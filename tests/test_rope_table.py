"""What make_rope takes for a table: the kernels read it by its address, so that one in host memory must not get there."""
import pytest
import torch

from paper_2508_15919_amd import binding as hb


def test_a_table_in_host_memory_is_refused():
    for rows in (0, 1, 8):
        with pytest.raises(ValueError, match="GPU"):
            hb.make_rope(torch.zeros(rows, 64), 64)


@pytest.mark.gpu
def test_a_table_on_the_gpu_is_taken():
    table = torch.zeros(8, 64, device="cuda")
    rope = hb.make_rope(table, 64, True)
    assert (rope.cos_sin, rope.num_positions, rope.rot_dim, rope.interleaved) == (table.data_ptr(), 8, 64, 1) and rope.table is table
    with pytest.raises(ValueError):
        hb.make_rope(table.double(), 64)
