"""Block tables that the bindings refuse, without a GPU: a slice of a wider table, whose rows lie further apart than the library is told."""
import pytest
import torch

from paper_2608_26523_b200 import api

bf16 = torch.bfloat16
x, freq, lens = torch.zeros(5, 4, 128, dtype=bf16), torch.ones(32), torch.zeros(2, dtype=torch.int32)
cache, means, lists = torch.zeros(8, 16, 4, 128, dtype=bf16), torch.zeros(8, 4, 128, dtype=bf16), torch.zeros(5, 4, 8, dtype=torch.int32)
workspace = torch.zeros(256, dtype=torch.uint8)
CALLS = {
    "append": lambda table: api.vpp_kv_append_rope(x, x, cache, cache, table, lens, lens, 16, 64, freq),
    "means": lambda table: api.vpp_block_means(cache, means, table, lens, lens, 16, 5),
    "select": lambda table: api.vpp_block_select(x, means, table, lens, lens, 16, 64, lists, workspace),
    "attention": lambda table: api.make_args(x, cache, cache, table, lens, lens, 16, 64, 1.0),
}


@pytest.mark.parametrize("call", CALLS)
def test_a_slice_of_a_wider_table(call):
    with pytest.raises(AssertionError):
        CALLS[call](torch.zeros(2, 9, dtype=torch.int32)[:, :4])
    with pytest.raises(AssertionError):
        CALLS[call](torch.zeros(4, 2, dtype=torch.int32).t())


def test_dense_tables():
    wide = torch.zeros(1, 9, dtype=torch.int32)
    for table in (torch.zeros(2, 4, dtype=torch.int32), wide[:, :4], None):
        assert api.make_args(x, cache, cache, table, lens, lens, 16, 64, 1.0).max_blocks_per_req == (0 if table is None else 4)
