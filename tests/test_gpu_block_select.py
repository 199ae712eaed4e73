"""vpp_block_means and vpp_block_select against the fp64 oracle.  Lists are equal, not close."""
import numpy as np
import pytest
import torch

from block_parity import f64, generator, ints, randn
from oracle.ref_block_sparse import completed_pages, ref_block_means, ref_block_select
from paper_2608_26523_b200 import api

pytestmark = pytest.mark.gpu


def paged(gen, prefix, chunk, page):
    R, width = len(prefix), max(1, max(-(-(p + c) // page) for p, c in zip(prefix, chunk)))
    pool = R * width + 2
    return torch.randperm(pool, generator=gen, device="cuda")[:R * width].to(torch.int32).view(R, width), pool


# ---- means ----------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("page", [1, 2, 16, 32, 64, 128, 512])
@pytest.mark.parametrize("prefix, chunk, hkv", [([0], [1], 1), ([15, 16, 0, 100, 31], [1, 15, 300, 0, 130], 2), ([777], [1500], 8),
                                                ([i * 7 for i in range(150)], [1] * 150, 3)])
def test_means(page, prefix, chunk, hkv):
    gen = generator(page)
    table, pool = paged(gen, prefix, chunk, page)
    k = randn(gen, pool, page, hkv, 128) + randn(gen, pool, 1, hkv, 128)
    means = torch.full((pool, hkv, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    status = ints([-1])
    api.vpp_block_means(k, means, table, ints(prefix), ints(chunk), page, sum(chunk), status=status)
    assert int(status) == 0
    want = ref_block_means(f64(k), table.cpu().numpy(), prefix, chunk, page)
    got, mag = f64(means), np.abs(f64(k)).mean(axis=1)
    for b in range(pool):
        if b in want:     # rounded once (2^-8); sums of at most 512 terms in 32 bits
            assert (np.abs(got[b] - want[b]) <= 2.0 ** -8 * np.abs(want[b]) + 512 * 2.0 ** -24 * mag[b]).all()
        else:
            assert (got[b] == 9.0).all()


def test_means_of_a_strided_cache_past_32_bits():
    gen = generator(3)
    page, hkv = 64, 2
    pool = (9 << 30) // (page * hkv * 2 * 256)
    both = torch.zeros((pool, page, hkv, 256), dtype=torch.bfloat16, device="cuda")     # keys and values side by side
    table = ints([[pool - 1, 1, pool - 2]])
    both[table[0].long()] = randn(gen, 3, page, hkv, 256)
    means = torch.zeros((pool, hkv, 128), dtype=torch.bfloat16, device="cuda")
    api.vpp_block_means(both[..., :128], means, table, ints([0]), ints([192]), page, 192)
    want = f64(both[table[0].long()][..., :128]).mean(axis=1)
    assert np.allclose(f64(means[table[0].long()]), want, rtol=2.0 ** -8, atol=1e-5)
    assert int((means.view(pool, -1) != 0).any(1).sum()) == 3


def test_means_checks_on_the_device():
    gen = generator(4)
    table, pool = paged(gen, [30, 0], [40, 33], 16)
    k, means = randn(gen, pool, 16, 2, 128), torch.zeros((pool, 2, 128), dtype=torch.bfloat16, device="cuda")
    status = ints([0])
    for prefix, chunk in (([30, 0], [40, 32]), ([30, -1], [40, 33]), ([50, 0], [40, 33])):
        api.vpp_block_means(k, means, table, ints(prefix), ints(chunk), 16, 73, status=status)
        assert int(status) == 1 and (means == 0).all()
    wrong = table.clone()
    wrong[0, 3] = pool
    api.vpp_block_means(k, means, wrong, ints([30, 0]), ints([40, 33]), 16, 73, status=status)
    assert int(status) == 2
    done = {int(table[r, j]) for r, j in completed_pages([30, 0], [40, 33], 16)} - {int(table[0, 3])}
    assert {int(b) for b in (means.view(pool, -1) != 0).any(1).nonzero()} == done


# ---- selection ------------------------------------------------------------------------------------------------------------------

def select(q, means, table, prefix, chunk, page, topk, first, last, max_seq=None, want_status=0):
    T, hq, hkv = q.shape[0], q.shape[1], means.shape[1]
    max_seq = max(p + c for p, c in zip(prefix, chunk)) if max_seq is None else max_seq
    store = torch.full((T + 2, hkv, topk), -77, dtype=torch.int32, device="cuda")       # rows before and behind stay as they are
    ws = torch.empty(api.vpp_block_select_workspace_size(T, len(prefix), hq, hkv, page, max_seq), dtype=torch.uint8, device="cuda")
    ws.fill_(0xff)
    status = ints([-1])
    api.vpp_block_select(q, means, table, ints(prefix), ints(chunk), page, max_seq, store[1:T + 1], ws, num_first=first, num_last=last, status=status)
    assert int(status) == want_status
    assert (store[0] == -77).all() and (store[T + 1] == -77).all()
    return store[1:T + 1]


def check(q, means, table, prefix, chunk, page, topk, first, last, **kw):
    got = select(q, means, table, prefix, chunk, page, topk, first, last, **kw)
    want = ref_block_select(f64(q), f64(means), table.cpu().numpy(), prefix, chunk, page, topk, first, last)
    assert (got.cpu().numpy() == want).all(), np.argwhere(got.cpu().numpy() != want)[:5]


@pytest.mark.parametrize("prefix, chunk", [([0], [1]), ([5000], [1]), ([3000, 64, 0, 5000, 12], [3, 70, 0, 1, 200]), ([4000], [300]),
                                           ([100 * i + 900 for i in range(40)], [1] * 40), ([2000, 2000, 2000], [4, 5, 128])])
@pytest.mark.parametrize("hq, hkv, page, topk, first, last", [(4, 1, 16, 8, 1, 2), (8, 8, 16, 30, 0, 1), (15, 5, 32, 4, 2, 2), (64, 4, 64, 16, 1, 1),
                                                              (32, 2, 16, 200, 3, 5), (128, 1, 16, 1, 0, 1), (16, 2, 16, 129, 0, 1)])
def test_selection(prefix, chunk, hq, hkv, page, topk, first, last):
    gen = generator(hq + page + topk)
    table, pool = paged(gen, prefix, chunk, page)
    check(randn(gen, sum(chunk), hq, 128), randn(gen, pool, hkv, 128), table, prefix, chunk, page, topk, first, last)


@pytest.mark.parametrize("prefix, chunk", [([40000], [2]), ([30000, 41000], [40, 1])])
def test_long_contexts(prefix, chunk):
    gen = generator(8)
    table, pool = paged(gen, prefix, chunk, 16)
    check(randn(gen, sum(chunk), 16, 128), randn(gen, pool, 2, 128), table, prefix, chunk, 16, 64, 1, 2)


def test_several_slabs_of_tokens():
    """More scores than a slab of the workspace holds; two requests meet inside one."""
    prefix, chunk, page = [60000, 100], [1300, 400], 16
    gen = generator(9)
    table, pool = paged(gen, prefix, chunk, page)
    q, means = randn(gen, 1700, 8, 128), randn(gen, pool, 8, 128)
    assert api.vpp_block_select_workspace_size(1700, 2, 8, 8, page, 61300) < 1700 * 8 * 3832 * 4
    got = select(q, means, table, prefix, chunk, page, 12, 1, 1).cpu().numpy()
    pick = [0, 1, 5, 511, 512, 513, 700, 1023, 1024, 1299, 1300, 1301, 1500, 1699]
    for t in pick:
        r, p = (0, 60000 + t) if t < 1300 else (1, 100 + t - 1300)
        row = ref_block_select(f64(q[t:t + 1]), f64(means), table[r:r + 1].cpu().numpy(), [p], [1], page, 12, 1, 1)
        assert (got[t] == row[0]).all(), t


@pytest.mark.parametrize("chunk", [3, 40])
@pytest.mark.parametrize("kind", ["zero queries", "zero means", "one mean", "few means", "nearly equal", "opposite heads", "tiny", "huge"])
def test_ties_and_near_ties(kind, chunk):
    """Where scores in 32 bits cannot tell: equal pages, pages a last bit apart, heads that cancel, products below and above the range."""
    gen = generator(10)
    prefix, page, topk = [9000], 16, 20
    table, pool = paged(gen, prefix, [chunk], page)
    q, means = randn(gen, chunk, 8, 128), randn(gen, pool, 2, 128)
    if kind == "zero queries":
        q.zero_()
    elif kind == "zero means":
        means.zero_()
    elif kind == "one mean":
        means[:] = means[:1].clone()
    elif kind == "few means":
        means[:] = means[torch.arange(pool, device="cuda") % 5].clone()
    elif kind == "nearly equal":
        means[:] = means[:1].clone()
        means[:, :, 7] += (torch.randn((pool, 2), generator=gen, device="cuda") * 0.01).to(torch.bfloat16)
    elif kind == "opposite heads":
        q[:, 1::2] = -q[:, 0::2] * (1 + 2.0 ** -7)
        q *= 100
    elif kind == "tiny":
        q *= 1e-30
        means *= 1e-12
    elif kind == "huge":
        q *= 1e20
        means *= 1e19
    check(q, means, table, prefix, [chunk], page, topk, 1, 2)


@pytest.mark.parametrize("chunk", [2, 30])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_infinite_and_nan_scores(value, chunk):
    gen = generator(11)
    prefix, page = [5000], 16
    table, pool = paged(gen, prefix, [chunk], page)
    q, means = randn(gen, chunk, 4, 128), randn(gen, pool, 1, 128)
    some = table[0, torch.randperm(table.shape[1], generator=gen, device="cuda")[:90]].long()
    means[some, 0, 3] = value
    q[1, 2, 5] = value                                          # a token of its own, whose scores are all infinite or NaN
    check(q, means, table, prefix, [chunk], page, 24, 1, 1)


def test_pages_that_are_not_scored_may_hold_anything():
    """Means of the forced pages and of pages past the own one are not looked at where they could decide."""
    gen = generator(12)
    prefix, chunk, page = [1600], [20], 16
    table, pool = paged(gen, prefix, chunk, page)
    q, means = randn(gen, 20, 4, 128), randn(gen, pool, 1, 128)
    got = select(q, means, table, prefix, chunk, page, 10, 1, 3)
    poisoned = torch.full_like(means, float("nan"))
    inner = table[0, 1:table.shape[1] - 2].long()
    poisoned[inner] = means[inner]
    assert torch.equal(select(q, poisoned, table, prefix, chunk, page, 10, 1, 3), got)


def test_checks_on_the_device():
    gen = generator(13)
    prefix, chunk, page = [700, 30], [40, 9], 16
    table, pool = paged(gen, prefix, chunk, page)
    q, means = randn(gen, 49, 4, 128), randn(gen, pool, 2, 128)
    for p, c in (([700, 30], [40, 8]), ([700, -1], [40, 9]), ([720, 30], [40, 9])):
        got = select(q, means, table, p, c, page, 6, 1, 1, max_seq=740, want_status=1)
        assert (got == -77).all()
    wrong = table.clone()
    wrong[0, 7] = pool
    wrong[0, 9] = -5
    got = select(q, means, wrong, prefix, chunk, page, 6, 1, 1, want_status=2)
    assert ((got >= -1) & (got <= 740 // page)).all()
    select(q, means, table, prefix, chunk, page, 6, 1, 1)


def test_two_streams_and_a_graph():
    """Calls with workspaces of their own on two streams at once, and a captured one replayed over new queries."""
    gen = generator(14)
    prefix, chunk, page = [6000], [200], 16
    table, pool = paged(gen, prefix, chunk, page)
    p, c = ints(prefix), ints(chunk)
    sets = []
    for _ in range(2):
        q, means = randn(gen, 200, 8, 128), randn(gen, pool, 2, 128)
        out = torch.empty((200, 2, 16), dtype=torch.int32, device="cuda")
        ws = torch.empty(api.vpp_block_select_workspace_size(200, 1, 8, 2, page, 6200), dtype=torch.uint8, device="cuda")
        sets.append((q, means, out, ws, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for q, means, out, ws, stream in sets:
            with torch.cuda.stream(stream):
                api.vpp_block_select(q, means, table, p, c, page, 6200, out, ws, num_first=1)
    torch.cuda.synchronize()
    for q, means, out, ws, _ in sets:
        assert torch.equal(out, select(q, means, table, prefix, chunk, page, 16, 1, 1))
    q, means, out, ws, _ = sets[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.vpp_block_select(q, means, table, p, c, page, 6200, out, ws, num_first=1)
    q.copy_(randn(gen, 200, 8, 128))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, select(q, means, table, prefix, chunk, page, 16, 1, 1))


@pytest.mark.parametrize("hkv, topk", [(8, 200), (1, 256), (8, 90)])
def test_portions_of_a_long_chunk(hkv, topk):
    """Candidates of all tokens take more than a portion of the workspace; requests begin and end inside one, decode rows among them."""
    prefix, chunk, page = [60000, 100, 44444, 9000, 30000], [1300, 400, 1, 3, 2300 if hkv == 8 else 9000], 16
    T = sum(chunk)
    gen = generator(10)
    table, pool = paged(gen, prefix, chunk, page)
    q, means = randn(gen, T, 8, 128), randn(gen, pool, hkv, 128)
    got = select(q, means, table, prefix, chunk, page, topk, 1, 2).cpu().numpy()
    cu = np.concatenate([[0], np.cumsum(chunk)])
    m64, tab = f64(means), table.cpu().numpy()
    for t in sorted({0, 255, 256, 700, 767, 768, 1023, 1024, 1279, 1280, 1299, 1300, 1535, 1536, 1699, 1700, 1701, 1702, 1703, 1704, 2047, 2048, 2303, 2304, 3000, T - 1}):
        r = int(np.searchsorted(cu, t, side="right")) - 1
        row = ref_block_select(f64(q[t:t + 1]), m64, tab[r:r + 1], [prefix[r] + t - int(cu[r])], [1], page, topk, 1, 2)
        assert (got[t] == row[0]).all(), t


def test_no_more_tokens_than_requests_but_a_request_with_most_of_them():
    """Launches with places for requests that are not there: no request has a token but one, two or three."""
    page, n = 16, 260
    for at in ({17: 200}, {0: 100, 259: 1}, {3: 2, 4: 5, 258: 90}):
        prefix = [(37 * i) % 900 + 600 for i in range(n)]
        chunk = [at.get(i, 0) for i in range(n)]
        gen = generator(11)
        table, pool = paged(gen, prefix, chunk, page)
        check(randn(gen, sum(chunk), 8, 128), randn(gen, pool, 2, 128), table, prefix, chunk, page, 12, 1, 2)


@pytest.mark.parametrize("chunk", [[2, 1], [30, 3]])
@pytest.mark.parametrize("topk, first, last", [(256, 0, 1), (140, 3, 2)])
def test_more_listed_by_the_runs_than_is_gathered_at_a_time(chunk, topk, first, last):
    """Rows of more than 8192 pages: three runs, each of which lists `topk` and more."""
    prefix = [140000, 131050]
    gen = generator(12)
    table, pool = paged(gen, prefix, chunk, 16)
    check(randn(gen, sum(chunk), 4, 128), randn(gen, pool, 1, 128), table, prefix, chunk, 16, topk, first, last)
