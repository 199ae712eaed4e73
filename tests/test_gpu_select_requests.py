"""vpp_block_select of launches with as many requests as its documentation allows, chunks among them."""
import numpy as np
import pytest
import torch

from block_parity import f64, generator, ints, randn
from oracle.ref_block_sparse import ref_block_select
from paper_2608_26523_b200 import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R", [1790, 1800, 4097, 8192])
def test_chunks_among_thousands_of_requests(R):
    """Contexts of up to 4095 pages (the longest run of an item): decode rows, requests without tokens, three chunks."""
    page, topk, first, last, pool, most = 16, 24, 1, 2, 5000, 65520
    gen, rng = generator(R), np.random.default_rng(R)
    prefix, chunk = rng.integers(0, 300, R), (rng.random(R) > 0.03).astype(int)      # (more tokens than requests: not all are decode rows)
    for r, p, c in ((0, 65000, 5), (R // 2, 40000, 300), (R - 1, most - 130, 130), (7, 30000, 1), (R - 3, 60000, 4)):
        prefix[r], chunk[r] = p, c
    T = int(chunk.sum())
    assert T > R
    table = torch.randint(0, pool, (R, most // page), generator=gen, device="cuda", dtype=torch.int32)       # (requests may share pages)
    q, means = randn(gen, T, 4, 128), randn(gen, pool, 1, 128)
    ws = torch.empty(api.vpp_block_select_workspace_size(T, R, 4, 1, page, most), dtype=torch.uint8, device="cuda").fill_(255)
    got, status = torch.full((T, 1, topk), -77, dtype=torch.int32, device="cuda"), ints([-1])
    api.vpp_block_select(q, means, table, ints(prefix.tolist()), ints(chunk.tolist()), page, most, got, ws, num_first=first, num_last=last, status=status)
    assert int(status) == 0
    got, m64, q64 = got.cpu().numpy(), f64(means), f64(q)
    cu = np.concatenate([[0], np.cumsum(chunk)])
    rows = {t for r in (0, 7, R // 2, R - 3, R - 1) for t in list(range(cu[r], cu[r + 1]))[::7] + [cu[r + 1] - 1]} | set(range(0, T, 97))
    for t in sorted(rows):
        r = int(np.searchsorted(cu, t, side="right")) - 1
        want = ref_block_select(q64[t:t + 1], m64, table[r:r + 1].cpu().numpy(), [int(prefix[r]) + t - int(cu[r])], [1], page, topk, first, last)
        assert (got[t] == want[0]).all(), (t, r)


@pytest.mark.parametrize("prefix, chunk", [([900, 0, 333], [1, 1, 1]), ([900, 0, 333], [300, 20, 1]), ([3000], [4])])
@pytest.mark.parametrize("topk, first", [(1, 0), (4, 2), (200, 3)])
def test_lists_by_position_alone(prefix, chunk, topk, first):
    """num_first + num_last = topk: no page is scored, so no query, mean or page of the table is looked at, and the workspace holds nothing."""
    page, T = 16, sum(chunk)
    most = max(p + c for p, c in zip(prefix, chunk))
    nothing = torch.full((T, 4, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    table = torch.full((len(prefix), -(-most // page)), -1, dtype=torch.int32, device="cuda")
    means = torch.full((3, 2, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(api.vpp_block_select_workspace_size(T, len(prefix), 4, 2, page, most, topk, first, topk - first), dtype=torch.uint8, device="cuda")
    got = torch.full((T + 1, 2, topk), -77, dtype=torch.int32, device="cuda")
    for c, want in ((chunk, 0), ([chunk[0] + 1] + chunk[1:], 1), (chunk, 0)):
        status = ints([-1])
        api.vpp_block_select(nothing, means, table, ints(prefix), ints(c), page, most + 1, got[:T], ws, num_first=first, num_last=topk - first, status=status)
        assert int(status) == want
        if want:
            assert (got == -77).all()
        else:
            lists = ref_block_select(np.zeros((T, 4, 128)), np.zeros((1, 2, 128)), np.zeros(table.shape, np.int64), prefix, c, page, topk, first, topk - first)
            assert (got[:T].cpu().numpy() == lists).all() and (got[T] == -77).all()
            got.fill_(-77)
