"""The calls of a block-sparse layer as they are used: a prompt in chunks, then decode steps, of several requests at once --
vpp_kv_append_rope, vpp_block_means, vpp_block_select, vpp_block_attn_fwd -- with every step held to the oracles."""
import numpy as np
import pytest
import torch

from block_parity import block_args, check_attn, f64, generator, ints, randn
from oracle.ref_block_sparse import ref_block_attn, ref_block_select, ref_rope, rows_of
from paper_2608_26523_b200 import api, workloads as W

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq, hkv, page, topk", [(8, 2, 16, 6), (15, 5, 32, 3), (16, 1, 64, 4)])
def test_prompts_in_chunks_then_decode_steps(hq, hkv, page, topk):
    gen = generator(hq)
    steps = [([0, 0, 0], [150, 33, 0]), ([150, 33, 0], [200, 100, 90]), ([350, 133, 90], [1, 77, 1]), ([351, 210, 91], [1, 1, 1]), ([352, 211, 92], [1, 1, 1])]
    R, width, most = 3, -(-353 // page), 353
    pool = R * width + 2
    table = torch.randperm(pool, generator=gen, device="cuda")[:R * width].to(torch.int32).view(R, width)
    nan = lambda *s: torch.full(s, float("nan"), dtype=torch.bfloat16, device="cuda")      # noqa: E731
    k_cache, v_cache, means = nan(pool, page, hkv, 128), nan(pool, page, hkv, 128), nan(pool, hkv, 128)
    f = torch.tensor(10000.0 ** (-np.arange(64) / 64), dtype=torch.float32, device="cuda")
    keys = [np.zeros((most, hkv, 128)) for _ in range(R)]           # the rotated keys as the oracle has them
    for prefix, chunk in steps:
        T = sum(chunk)
        qkv = randn(gen, T, hq + 2 * hkv, 128)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        q_rot = torch.empty((T, hq, 128), dtype=torch.bfloat16, device="cuda")
        p, c, status = ints(prefix), ints(chunk), ints([-1])
        api.vpp_kv_append_rope(k, v, k_cache, v_cache, table, p, c, page, most, f, q=q, q_out=q_rot, status=status)
        assert int(status) == 0
        rows = rows_of(prefix, chunk)
        pos = [x for _, x in rows]
        turned = ref_rope(f64(k), pos, f.cpu().numpy().astype(np.float64))
        for i, (r, x) in enumerate(rows):
            keys[r][x] = turned[i]
            assert torch.equal(v_cache[int(table[r, x // page]), x % page], v[i])
        assert np.abs(f64(q_rot) - ref_rope(f64(q), pos, f.cpu().numpy().astype(np.float64))).max() <= 2.0 ** -8 * 8

        api.vpp_block_means(k_cache, means, table, p, c, page, T, status=status)
        assert int(status) == 0
        for r in range(R):
            full = (prefix[r] + chunk[r]) // page
            for j in range(full):          # those of earlier steps are still there
                mine = keys[r][j * page:(j + 1) * page]
                # (keys rounded to 2^-8, the mean of theirs, rounded again)
                assert (np.abs(f64(means[int(table[r, j])]) - mine.mean(0)) <= 2.0 ** -8 * (np.abs(mine).mean(0) + np.abs(mine.mean(0))) + 1e-5).all()
            for j in range(full, width):
                assert torch.isnan(means[int(table[r, j])]).all()

        lists = torch.empty((T, hkv, topk), dtype=torch.int32, device="cuda")
        ws = torch.empty(api.vpp_block_select_workspace_size(T, R, hq, hkv, page, most), dtype=torch.uint8, device="cuda")
        api.vpp_block_select(q_rot, means, table, p, c, page, most, lists, ws, num_first=1, num_last=1, status=status)
        assert int(status) == 0
        want = ref_block_select(f64(q_rot), f64(means), table.cpu().numpy(), prefix, chunk, page, topk, 1, 1)
        assert (lists.cpu().numpy() == want).all()

        prob = W.Problem(q=q_rot, k_cache=k_cache, v_cache=v_cache, block_table=table, prefix_len=p, chunk_len=c, block_size=page, max_seq_len=most,
                         num_q_heads=hq, num_kv_heads=hkv, head_dim_qk=128, head_dim_v=128, scale=128 ** -0.5)
        a, out, lse, status = block_args(prob, lists)
        api.vpp_block_attn_fwd(a, lists)
        assert int(status) == 0
        check_attn(out, lse, ref_block_attn(f64(q_rot), np.nan_to_num(f64(k_cache)), np.nan_to_num(f64(v_cache)), want, table.cpu().numpy(), prefix, chunk,
                                            page, 128 ** -0.5))


def test_the_chain_captured_in_one_graph():
    """All four calls in one graph, replayed for three decode steps whose lengths and rows change in place."""
    gen = generator(77)
    hq, hkv, page, topk, R, most = 8, 2, 16, 5, 4, 400
    pool = R * 25
    table = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32).view(R, 25)
    k_cache, v_cache = randn(gen, pool, page, hkv, 128), randn(gen, pool, page, hkv, 128)
    means = torch.zeros((pool, hkv, 128), dtype=torch.bfloat16, device="cuda")
    f = torch.tensor(10000.0 ** (-np.arange(64) / 64), dtype=torch.float32, device="cuda")
    start = [381, 79, 160, 15]
    api.vpp_block_means(k_cache, means, table, ints([0] * R), ints(start), page, sum(start))
    p, c, qkv = ints(start), ints([1] * R), randn(gen, R, hq + 2 * hkv, 128)
    q_rot, lists = torch.empty((R, hq, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((R, hkv, topk), dtype=torch.int32, device="cuda")
    ws = torch.empty(api.vpp_block_select_workspace_size(R, R, hq, hkv, page, most), dtype=torch.uint8, device="cuda")
    prob = W.Problem(q=q_rot, k_cache=k_cache, v_cache=v_cache, block_table=table, prefix_len=p, chunk_len=c, block_size=page, max_seq_len=most,
                     num_q_heads=hq, num_kv_heads=hkv, head_dim_qk=128, head_dim_v=128, scale=128 ** -0.5)
    a, out, lse, status = block_args(prob, lists)
    caches = [t.clone() for t in (k_cache, v_cache, means)]

    def step():
        api.vpp_kv_append_rope(qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], k_cache, v_cache, table, p, c, page, most, f, q=qkv[:, :hq], q_out=q_rot)
        api.vpp_block_means(k_cache, means, table, p, c, page, R)
        api.vpp_block_select(q_rot, means, table, p, c, page, most, lists, ws, num_first=1, num_last=1)
        api.vpp_block_attn_fwd(a, lists)

    rows = [randn(gen, R, hq + 2 * hkv, 128) for _ in range(3)]
    want = []
    for i in range(3):
        qkv.copy_(rows[i])
        p.copy_(ints([x + i for x in start]))
        step()
        want.append((out.clone(), lse.clone(), lists.clone()))
    for t, was in zip((k_cache, v_cache, means), caches):
        t.copy_(was)
    p.copy_(ints(start))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        qkv.copy_(rows[i])
        p.copy_(ints([x + i for x in start]))
        graph.replay()
        torch.cuda.synchronize()
        assert int(status) == 0
        assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1]) and torch.equal(lists, want[i][2])
