"""Calls of two host threads at a time, one with large shapes and one with small ones: neither may change what the other's launches need."""
import threading

import numpy as np
import pytest
import torch

from block_parity import block_args, generator, ints, randn
from paper_2608_26523_b200 import api, workloads as W

pytestmark = pytest.mark.gpu


def together(calls, rounds):
    """Every call `rounds` times in a thread and on a stream of its own; the errors."""
    gate, errors = threading.Barrier(len(calls)), []

    def work(call):
        stream = torch.cuda.Stream()
        gate.wait()
        for _ in range(rounds):
            try:
                call(stream.cuda_stream)
            except api.VppError as e:
                errors.append(str(e))
        stream.synchronize()

    threads = [threading.Thread(target=work, args=(c,)) for c in calls]
    torch.cuda.synchronize()
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    return errors


def selection(seed, R, chunk, pages):
    """A selection of R requests of `chunk` tokens, contexts of `pages` pages of 16; what it lists alone and in `call`."""
    gen, page, topk = generator(seed), 16, 20
    prefix, most, T, pool = [pages * 16 - chunk] * R, pages * 16, R * chunk, pages + 9
    table = torch.randint(0, pool, (R, pages), generator=gen, device="cuda", dtype=torch.int32)
    q, means = randn(gen, T, 4, 128), randn(gen, pool, 1, 128)
    size = api.vpp_block_select_workspace_size(T, R, 4, 1, page, most)
    p, c = ints(prefix), ints([chunk] * R)
    sets = [(torch.full((T, 1, topk), -77, dtype=torch.int32, device="cuda"), torch.empty(size, dtype=torch.uint8, device="cuda"), ints([-1])) for _ in range(2)]

    def call(out, ws, status, stream=None):
        api.vpp_block_select(q, means, table, p, c, page, most, out, ws, num_first=1, status=status, stream=stream)
    call(*sets[0])
    return (lambda stream: call(*sets[1], stream)), sets[0][0], sets[1][0], sets[1][2]


@pytest.mark.parametrize("chunk", [1, 5])
def test_selection(chunk):
    """Different requests (their lengths are in shared memory) and runs of pages: decode rows, and chunks."""
    got = [selection(1, 700, chunk, 4000), selection(2, 2, chunk, 150)]
    assert together([g[0] for g in got], 400) == []
    for _, want, out, status in got:
        assert int(status) == 0 and torch.equal(out, want)


def test_attention_over_listed_pages():
    got = []
    for seed, R, most in ((3, 8000, 64), (4, 2, 2000)):
        page, hkv, topk = 16, 1, 4
        rng = np.random.default_rng(seed)
        prob = W.make_problem(seed, rng.integers(0, most - 3, R).tolist(), [2] * R, 4, hkv, 128, 128, block_size=page).to("cuda")
        lists = torch.from_numpy(rng.integers(-1, most // page, (2 * R, hkv, topk)).astype(np.int32)).cuda()
        a, want, want_lse, _ = block_args(prob, lists)
        api.vpp_block_attn_fwd(a, lists)
        b, out, lse, status = block_args(prob, lists)
        got.append((lambda stream, b=b, lists=lists: api.vpp_block_attn_fwd(b, lists, stream=stream), want, out, status, a, prob))
    assert together([g[0] for g in got], 400) == []
    for _, want, out, status, *_ in got:
        assert int(status) == 0 and torch.equal(out, want)
