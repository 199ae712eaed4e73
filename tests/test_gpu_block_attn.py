"""vpp_block_attn_fwd against the fp64 oracle, every element."""
import numpy as np
import pytest
import torch

from block_parity import block_args, check_attn, f64, generator, ints, randn
from oracle.ref_block_sparse import ref_block_attn, rows_of
from paper_2608_26523_b200 import api, workloads as W

pytestmark = pytest.mark.gpu


def make_lists(seed, prefix, chunk, hkv, topk, page, kind="mixed"):
    """Lists of every sort: shared by neighbours, independent, with padding, duplicates, pages ahead and other values that are no page, empty ones."""
    rng = np.random.default_rng(seed)
    rows = rows_of(prefix, chunk)
    out = np.full((len(rows), hkv, topk), -1, np.int32)
    shared = {}
    for t, (r, p) in enumerate(rows):
        c = p // page
        for g in range(hkv):
            how = kind if kind != "mixed" else ["shared", "shared", "shared", "own", "free", "odd", "empty"][rng.integers(7)]
            if how == "empty":
                out[t, g] = rng.integers(-5, 0, topk) if rng.integers(2) else c + 1 + rng.integers(0, 99, topk)
            elif how == "own":
                out[t, g, 0] = c
            elif how == "odd":
                out[t, g] = rng.integers(-3, c + 4, topk)
                out[t, g, -1] = -2 ** 31 if rng.integers(2) else 2 ** 31 - 1
            else:
                key = (r, g, t // 16 if how == "shared" else t)
                if key not in shared:
                    shared[key] = rng.permutation(c + 1)[:topk]
                pages = np.unique(np.concatenate([[0, c], shared[key]]))[-topk:]
                out[t, g, :len(pages)] = pages
                rng.shuffle(out[t, g])
    return out


def run(prob_cpu, lists, splits=0, label="", prob_gpu=None):
    prob = prob_cpu.to("cuda") if prob_gpu is None else prob_gpu
    T, hq = prob.total_q, prob.num_q_heads
    out = torch.full((T + 2, hq, 128), float("nan"), dtype=torch.bfloat16, device="cuda")       # rows before and behind stay as they are
    lse = torch.full((T + 2, hq), float("nan"), device="cuda")
    dev = torch.from_numpy(lists).cuda()
    a, _, _, status = block_args(prob, dev, splits, out[1:T + 1], lse[1:T + 1])
    api.vpp_block_attn_fwd(a, dev)
    torch.cuda.synchronize()
    assert int(status) == 0, label
    for x in (out, lse):
        assert torch.isnan(x[0]).all() and torch.isnan(x[T + 1]).all()
    # (unused pages and slots past the end hold NaN: zeros for the oracle, which does not look at them but multiplies whole arrays)
    kc, vc = (np.nan_to_num(f64(c)) for c in (prob_cpu.k_cache, prob_cpu.v_cache))
    want = ref_block_attn(f64(prob_cpu.q), kc, vc, lists, prob_cpu.block_table.numpy(), prob_cpu.prefix_len.numpy(), prob_cpu.chunk_len.numpy(),
                          prob_cpu.block_size, prob_cpu.scale)
    check_attn(out[1:T + 1], lse[1:T + 1], want, label)
    return out[1:T + 1]


def problem(seed, prefix, chunk, hq, hkv, page):
    return W.make_problem(seed, prefix, chunk, hq, hkv, 128, 128, block_size=page, std=0.8)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("hq, hkv", [(1, 1), (4, 1), (16, 2), (15, 5), (64, 4), (6, 6), (48, 2), (128, 1), (8, 4)])
@pytest.mark.parametrize("splits", [0, 1, 3])
def test_lists_of_every_sort(page, hq, hkv, splits):
    prefix, chunk = [300, 0, 1000, 77, 15, 640], [9, 1, 0, 40, 1, 21]
    prob = problem(page + hq, prefix, chunk, hq, hkv, page)
    run(prob, make_lists(page * hq + splits, prefix, chunk, hkv, 7, page), splits, "page %d heads %d/%d splits %d" % (page, hq, hkv, splits))


@pytest.mark.parametrize("prefix, chunk, topk", [([0], [1], 1), ([0], [2], 1), ([1], [1], 1), ([16], [1], 3), ([127], [1], 40), ([128], [129], 9), ([4095], [1], 64),
                                                 ([0, 0, 0], [130, 1, 127], 12), ([5000], [257], 33), ([700] * 40, [1] * 40, 8)])
@pytest.mark.parametrize("page", [16, 128])
def test_lengths(prefix, chunk, topk, page):
    prob = problem(sum(prefix) + topk, prefix, chunk, 16, 2, page)
    run(prob, make_lists(7, prefix, chunk, 2, topk, page, "shared"), 0, "shared")
    run(prob, make_lists(8, prefix, chunk, 2, topk, page), 0, "mixed")


@pytest.mark.parametrize("splits", [2, 16, 64])
def test_more_parts_than_steps(splits):
    prefix, chunk = [900, 10, 500], [1, 1, 3]
    prob = problem(40 + splits, prefix, chunk, 8, 2, 64)
    lists = make_lists(splits, prefix, chunk, 2, 16, 64, "shared")
    lists[1] = -1
    run(prob, lists, splits)


def test_every_page_listed_is_dense_attention():
    prefix, chunk, page = [517, 0], [200, 90], 64
    prob = problem(51, prefix, chunk, 16, 2, page)
    width = prob.block_table.shape[1]
    lists = np.broadcast_to(np.arange(width, dtype=np.int32)[::-1], (290, 2, width)).copy()
    out = run(prob, lists)
    dense, _ = api.ChunkAttn(prob.to("cuda")).run()
    assert float((dense.float() - out.float()).abs().max()) <= 2e-2      # (two results within 1e-2 of the oracle)


def test_many_tokens_and_unions_of_many_windows():
    """Contexts of more pages than a window of the union's bitmap, at the largest mask (one q-head a kv-head) and the smallest."""
    for hq, hkv, prefix, chunk in ((1, 1, 40000, 130), (8, 1, 139990, 20)):
        prob = problem(60 + hq, [prefix], [chunk], hq, hkv, 16)
        lists = make_lists(61, [prefix], [chunk], hkv, 24, 16, "free")
        run(prob, lists, 0, "%d heads" % hq)


def test_strided_caches():
    """Keys and values side by side in one allocation, padded rows, heads before slots."""
    prefix, chunk, page = [300, 64], [50, 3], 32
    prob = problem(70, prefix, chunk, 12, 3, page)
    lists = make_lists(71, prefix, chunk, 3, 6, page)
    gpu = prob.to("cuda")
    nb, bs, h, d = gpu.k_cache.shape
    store = torch.full((nb, bs, h, 2 * d + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    store[..., :d], store[..., d + 8:] = gpu.k_cache, gpu.v_cache
    gpu.k_cache, gpu.v_cache = store[..., :d], store[..., d + 8:]
    one = run(prob, lists, 0, "side by side", gpu)
    heads = prob.to("cuda")
    for name in ("k_cache", "v_cache"):
        setattr(heads, name, getattr(heads, name).transpose(1, 2).contiguous().transpose(1, 2))
    assert torch.equal(one, run(prob, lists, 0, "heads before slots", heads))
    assert torch.equal(one, run(prob, lists, 0, "plain"))


def test_pages_past_32_bits_and_past_one_coordinate():
    prefix, chunk = [40], [60]
    prob = W.make_problem(80, prefix, chunk, 4, 2, 128, 128, block_size=64, std=0.8, pool_factor=1.0)
    lists = make_lists(81, prefix, chunk, 2, 2, 64)
    gpu = prob.to("cuda")
    nb, bs, h, d = gpu.k_cache.shape
    for far in ((3 << 30), 18 * (1 << 30) + 8):          # elements between pages; the second with hardly a divisor in common with a head
        if torch.cuda.mem_get_info()[0] < far * 2 * (nb - 1) + (1 << 30):
            pytest.skip("needs a cache of %d GB" % (far * 2 * (nb - 1) >> 30))
        store = torch.empty((nb - 1) * far + bs * h * d, dtype=torch.bfloat16, device="cuda")
        view = store.as_strided(gpu.k_cache.shape, (far, h * d, d, 1))
        view.copy_(prob.k_cache)
        far_gpu = prob.to("cuda")
        far_gpu.k_cache = view
        run(prob, lists, 0, "keys far apart", far_gpu)
        view.copy_(prob.v_cache)
        far_gpu = prob.to("cuda")
        far_gpu.v_cache = view
        run(prob, lists, 0, "values far apart", far_gpu)
        del store, view, far_gpu


def test_poison_where_nobody_looks():
    """Infinite and NaN keys in a page that neighbours list touch those that list it only; pages nobody lists may hold anything."""
    prefix, chunk, page = [500], [24], 16
    prob = problem(90, prefix, chunk, 8, 1, page)
    lists = make_lists(91, prefix, chunk, 1, 6, page, "shared")
    lists[lists == 3] = -1
    lists[5, 0] = [3, 0, 1, 2, 20, -1]
    clean = run(prob, lists)
    gpu = prob.to("cuda")
    gpu.k_cache[prob.block_table[0, 3].item(), 2] = float("nan")
    gpu.k_cache[prob.block_table[0, 3].item(), 7] = float("inf")
    dev = torch.from_numpy(lists).cuda()
    a, out, lse, status = block_args(gpu, dev)
    api.vpp_block_attn_fwd(a, dev)
    assert int(status) == 0 and torch.isnan(out[5]).all() and torch.isnan(lse[5]).all()
    rest = torch.arange(24) != 5
    assert torch.equal(out[rest], clean[rest])
    lists[5, 0, 0] = -1                       # now nobody lists the page
    clean = run(prob, lists)                  # (another union: other steps, other roundings)
    gpu.v_cache[prob.block_table[0, 3].item()] = float("nan")
    dev = torch.from_numpy(lists).cuda()
    a, out, lse, status = block_args(gpu, dev)
    api.vpp_block_attn_fwd(a, dev)
    assert torch.equal(out, clean)


def test_large_scores():
    """Scores of thousands: the running maximum moves by far more than the rescale threshold, in every order of pages."""
    prefix, chunk, page = [600], [33], 16
    prob = problem(95, prefix, chunk, 4, 2, page)
    steps = torch.arange(prob.k_cache.shape[0], dtype=torch.float32)[:, None, None, None] % 7 * 4 + 1
    prob.k_cache = (prob.k_cache.float() * steps).to(torch.bfloat16)
    prob.scale = 1.0
    run(prob, make_lists(96, prefix, chunk, 2, 20, page, "shared"), 0)


def test_checks_on_the_device():
    prefix, chunk, page = [100, 30], [20, 9], 16
    prob = problem(100, prefix, chunk, 4, 2, page).to("cuda")
    lists = torch.from_numpy(make_lists(101, prefix, chunk, 2, 4, page, "shared")).cuda()
    for p, c in (([100, 30], [20, 8]), ([100, -1], [20, 9]), ([120, 30], [20, 9])):
        for splits in (1, 2):
            bad = problem(100, prefix, chunk, 4, 2, page).to("cuda")
            bad.prefix_len, bad.chunk_len = ints(p), ints(c)
            a, out, lse, status = block_args(prob, lists, splits)
            a.prefix_len, a.chunk_len = bad.prefix_len.data_ptr(), bad.chunk_len.data_ptr()
            api.vpp_block_attn_fwd(a, lists)
            assert int(status) == 1 and torch.isnan(out).all() and torch.isnan(lse).all()
    a, out, lse, status = block_args(prob, lists)
    api.vpp_block_attn_fwd(a, lists)
    clean = out.clone()
    assert int(status) == 0
    wrong = prob.block_table.clone()
    wrong[0, 0] = prob.k_cache.shape[0]
    lists[:20, :, 0] = 0
    a, out, lse, status = block_args(prob, lists)
    a.block_table = wrong.data_ptr()
    api.vpp_block_attn_fwd(a, lists)
    assert int(status) == 2 and torch.equal(out[20:], clean[20:])


def test_same_bits_every_time_on_two_streams_and_replayed():
    prefix, chunk, page = [3000, 5, 700], [150, 1, 1], 64
    prob = problem(110, prefix, chunk, 64, 4, page).to("cuda")
    lists = torch.from_numpy(make_lists(111, prefix, chunk, 4, 12, page)).cuda()
    a, want, want_lse, _ = block_args(prob, lists)
    api.vpp_block_attn_fwd(a, lists)
    sets = [block_args(prob, lists) for _ in range(3)]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(10):
        for (b, *_), stream in zip(sets, streams):
            with torch.cuda.stream(stream):
                api.vpp_block_attn_fwd(b, lists)
    torch.cuda.synchronize()
    for _, out, lse, status in sets:
        assert int(status) == 0 and torch.equal(out, want) and torch.equal(lse, want_lse)
    b, out, lse, status = sets[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.vpp_block_attn_fwd(b, lists)
    lists.copy_(torch.from_numpy(make_lists(112, prefix, chunk, 4, 12, page)))
    graph.replay()
    torch.cuda.synchronize()
    got = out.clone()
    a, want, _, _ = block_args(prob, lists)
    api.vpp_block_attn_fwd(a, lists)
    assert torch.equal(got, want)


def test_two_calls_one_after_the_other_in_one_workspace():
    prefix, chunk, page = [900], [70], 32
    prob = problem(120, prefix, chunk, 8, 2, page)
    one, two = (make_lists(s, prefix, chunk, 2, 9, page) for s in (121, 122))
    want = [run(prob, x) for x in (one, two)]
    gpu = prob.to("cuda")
    d1, d2 = torch.from_numpy(one).cuda(), torch.from_numpy(two).cuda()
    a, out, _, _ = block_args(gpu, d1)
    b, out2, _, _ = block_args(gpu, d2)
    b.workspace, b.workspace_bytes = a.workspace, a.workspace_bytes
    for _ in range(3):
        api.vpp_block_attn_fwd(a, d1)
        api.vpp_block_attn_fwd(b, d2)
    assert torch.equal(out, want[0]) and torch.equal(out2, want[1])
