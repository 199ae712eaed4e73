"""vpp_block_select of one long chunk whose tokens take several portions of the workspace, the last of them with a few tokens only.  Lists are equal to
the fp64 oracle's, whatever the workspace held."""
import numpy as np
import pytest
import torch

from block_parity import f64, generator, ints, randn
from oracle.ref_block_sparse import ref_block_select
from paper_2608_26523_b200 import api

pytestmark = pytest.mark.gpu

FIRST, LAST = 1, 2


def check(seed, prefix, T, hq, hkv, page, topk, max_seq, fill, rows, calls=1):
    gen = generator(seed)
    width = -(-max_seq // page)
    pool = width + 3
    table = torch.randperm(pool, generator=gen, device="cuda")[:width].to(torch.int32).view(1, width)
    q, means = randn(gen, T, hq, 128), randn(gen, pool, hkv, 128)
    size = api.vpp_block_select_workspace_size(T, 1, hq, hkv, page, max_seq, topk, FIRST, LAST)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda").fill_(fill)
    got = torch.full((T, hkv, topk), -77, dtype=torch.int32, device="cuda")
    for _ in range(calls):
        status = ints([-1])
        api.vpp_block_select(q, means, table, ints([prefix]), ints([T]), page, max_seq, got, ws, num_first=FIRST, num_last=LAST, status=status)
        assert int(status) == 0
    got, m64, tab = got.cpu().numpy(), f64(means), table.cpu().numpy()
    for t in rows:
        want = ref_block_select(f64(q[t:t + 1]), m64, tab, [prefix + t], [1], page, topk, FIRST, LAST)
        assert (got[t] == want[0]).all(), t


@pytest.mark.parametrize("fill", [0, 255])
@pytest.mark.parametrize("rest", [0, 1, 2, 3, 4, 5])
@pytest.mark.parametrize("portions", [1, 3])
def test_far_into_a_prompt(rest, portions, fill):
    """Portions of 256 tokens (32 kv-heads, 2048 pages): the last tokens get lists of their own, not those of the tokens at the same place in the portion before."""
    T = 256 * portions + rest
    check(rest, 131072 - T, T, 32, 32, 64, 128, 131072, fill, [0, 1, 2, 3, 4, 255] + list(range(256 * portions, T)) + [T - 1])


@pytest.mark.parametrize("fill", [0, 255])
@pytest.mark.parametrize("rest", [1, 4, 5])
def test_from_the_start_of_a_prompt(rest, fill):
    """As above where the tokens at the same place in the portion before list all their pages: nothing of theirs is in the workspace."""
    T = 256 + rest
    check(10 + rest, 0, T, 32, 32, 1, 128, 20000, fill, [0, 3, 126, 127, 128, 129, 255] + list(range(256, T)), 2)


@pytest.mark.parametrize("T, hq, hkv, topk", [(7937, 64, 8, 32), (7940, 64, 8, 32), (1794, 64, 8, 128), (7683, 64, 4, 64)])
def test_long_chunks(T, hq, hkv, topk):
    """Portions of 7936, 1792 and 7680 tokens."""
    check(T, 131072 - T, T, hq, hkv, 64, topk, 131072, 255, [0, 1, 2, 3, 1791, 4000 % T] + list(range(T - 6, T)))
