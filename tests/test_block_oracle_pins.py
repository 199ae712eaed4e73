"""What the oracles of oracle/ref_block_sparse.py are held to: closed forms, identities and the dense oracle (CPU only)."""
import math

import numpy as np
import pytest

import oracle
from oracle.ref_block_sparse import completed_pages, ref_block_attn, ref_block_means, ref_block_select, ref_rope, rows_of
from oracle.ref_sparse_attn import bf16_bits_to_f64
from paper_2608_26523_b200 import workloads as W


def f64(t):
    return bf16_bits_to_f64(t.view(__import__("torch").int16).numpy())


def test_rotation_closed_forms():
    f = np.array([1.0, 0.25])
    x = np.array([[[1.0, 2.0, 3.0, 4.0]]])
    y = ref_rope(x, [2], f, "half")[0, 0]
    assert np.allclose(y, [math.cos(2) - 3 * math.sin(2), 2 * math.cos(.5) - 4 * math.sin(.5), 3 * math.cos(2) + math.sin(2), 4 * math.cos(.5) + 2 * math.sin(.5)])
    z = ref_rope(x, [2], f, "interleaved", amplitude=2.0)[0, 0]
    assert np.allclose(z, [2 * (math.cos(2) - 2 * math.sin(2)), 2 * (2 * math.cos(2) + math.sin(2)), 2 * (3 * math.cos(.5) - 4 * math.sin(.5)),
                           2 * (4 * math.cos(.5) + 3 * math.sin(.5))])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_identities(layout):
    rng = np.random.default_rng(1)
    f = 10000.0 ** (-np.arange(8) / 8)
    x, y = rng.standard_normal((1, 2, 24)), rng.standard_normal((1, 2, 24))
    a = ref_rope(x, [0], f, layout, 8)
    assert np.allclose(a, x)                                                         # position 0: nothing turns
    turn = lambda v, p: ref_rope(v, [p], f, layout, 8)                               # noqa: E731
    assert np.allclose(turn(x, 7)[..., :8], x[..., :8])                              # features outside stay
    assert np.allclose(turn(turn(x, 5), 6), turn(x, 11))                             # angles add up
    assert np.allclose((turn(x, 105) * turn(y, 103)).sum(-1), (turn(x, 2) * y)[..., 8:].sum(-1) + (x * y)[..., :8].sum(-1))      # only the distance counts
    assert np.allclose(np.linalg.norm(turn(x, 9)), np.linalg.norm(x))


def test_completed_pages():
    assert completed_pages([0, 15, 16, 31, 5], [16, 1, 15, 2, 0], 16) == [(0, 0), (1, 0), (3, 1)]
    k = np.arange(4 * 2 * 1 * 2, dtype=np.float64).reshape(4, 2, 1, 2)
    got = ref_block_means(k, np.array([[2, 0]]), [1], [2], 2)
    assert list(got) == [2] and np.allclose(got[2], (k[2, 0] + k[2, 1]) / 2)


def test_selection_by_hand():
    means = np.array([[[0.0]], [[5.0]], [[1.0]], [[5.0]], [[4.0]], [[float("nan")]], [[9.0]]])
    table = np.arange(7)[None]
    pick = lambda p, k, first, last: ref_block_select(np.ones((1, 1, 1)), means, table, [p], [1], 1, k, first, last)[0, 0].tolist()      # noqa: E731
    assert pick(2, 4, 0, 1) == [0, 1, 2, -1]             # fewer pages than topk
    assert pick(6, 2, 0, 1) == [1, 6]                    # a tie goes to the lowest page
    assert pick(6, 3, 1, 1) == [0, 1, 6]
    assert pick(6, 6, 1, 1) == [0, 1, 2, 3, 4, 6]        # NaN below everything
    assert pick(6, 4, 0, 2) == [1, 3, 5, 6]
    two = ref_block_select(np.array([[[1.0], [-3.0]]]), means, table, [4], [1], 1, 2, 0, 1)[0, 0].tolist()
    assert two == [0, 4]                                 # the heads of a group add up


def test_all_pages_listed_is_dense_attention():
    prob = W.make_problem(77, [37, 0, 90], [20, 9, 1], 4, 2, 128, 128, block_size=16, std=0.8, unused_fill=None, tail_fill=None)
    width = prob.block_table.shape[1]
    lists = np.broadcast_to(np.arange(width)[::-1], (prob.total_q, 2, width))
    out, lse, _ = ref_block_attn(f64(prob.q), f64(prob.k_cache), f64(prob.v_cache), lists, prob.block_table.numpy(), prob.prefix_len.numpy(),
                                 prob.chunk_len.numpy(), 16, prob.scale)
    rows = oracle.all_rows(prob.chunk_len.numpy(), 4)
    ref_o, ref_l = oracle.ref_chunk_attn_rows(prob.q, prob.k_cache, prob.v_cache, prob.k_cache.stride()[:3], prob.v_cache.stride()[:3],
                                              prob.block_table.numpy(), 16, prob.prefix_len.numpy(), prob.chunk_len.numpy(), 4, 2, 128, 128,
                                              prob.scale, rows)
    start = np.concatenate([[0], np.cumsum(prob.chunk_len.numpy())[:-1]])
    t = start[rows[:, 0]] + rows[:, 1]
    assert np.allclose(out[t, rows[:, 2]], ref_o, atol=1e-12) and np.allclose(lse[t, rows[:, 2]], ref_l, atol=1e-12)


def test_lists_are_sets_and_skip_what_is_no_page():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((2, 2, 4)), rng.standard_normal((3, 2, 1, 4)), rng.standard_normal((3, 2, 1, 4))
    run = lambda a, b: ref_block_attn(q, k, v, np.array([[a], [b]]), np.array([[2, 0, 1]]), [3], [2], 2, 0.5)      # noqa: E731
    one, two = run([0, 1, -1], [2, 0, -1]), run([1, 0, 0], [0, 2, 99])
    assert all(np.allclose(a, b) for a, b in zip(one, two))
    none = run([2, -1, -1], [-7, -1, 3])                 # page 2 lies ahead of position 3
    assert (none[0] == 0).all() and np.isneginf(none[1]).all()
    own = run([1, 1, 1], [2, 2, 2])
    assert np.allclose(own[0][1], np.broadcast_to(v[1, 0, 0], (2, 4)))      # position 4: one key of page 2
    assert rows_of([3], [2]) == [(0, 3), (0, 4)]
