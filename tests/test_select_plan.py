"""The host's plan of vpp_block_select, without a GPU: what its workspace has room for."""
import ctypes
import random

import pytest

from paper_2608_26523_b200 import api


@pytest.fixture(scope="module", autouse=True)
def lib():
    from paper_2608_26523_b200 import build
    build.build()                      # nvcc cross-compiles without a GPU
    return api.load_library()


@pytest.mark.parametrize("rest", [1, 2, 3, 4])
def test_a_last_portion_of_a_few_tokens_has_places_for_their_status(rest):
    """32 kv-heads, lists of 128 of 2048 pages: portions of 256 tokens.  Up to four tokens are scored by a kernel of their own, whose blocks have a word each."""
    size = lambda T: api.vpp_block_select_workspace_size(T, 1, 32, 32, 64, 131072, 128, 0, 1)      # noqa: E731
    assert size(256 + rest) >= size(256 + 5) + 4 * 32 * 4
    assert size(512 + rest + 5) == size(512 + 256)


def needed(T, R, hq, hkv, page, most, topk, first, last):
    """What the call itself asks for."""
    a = api.BlockSelectArgs(num_reqs=R, block_size=page, total_q=T, max_seq_len=most, num_q_heads=hq, num_kv_heads=hkv, head_dim=128, topk=topk, num_first=first,
                            num_last=last)
    return api.load_library().vpp_block_select_workspace_size(ctypes.byref(a))


def shapes():
    yield 175, 1, 1, 1, 32, 125237, 167, 1, 1
    yield 604, 1, 2, 2, 32, 126530, 70, 2, 2
    yield 1, 1, 64, 8, 64, 131072, 140, 0, 1
    yield 64, 1, 64, 8, 128, 131072, 130, 0, 1
    yield 300, 2, 64, 2, 64, 30000, 173, 1, 2
    rng = random.Random(5)
    log = lambda lo, hi: int(lo * (hi / lo) ** rng.random())      # noqa: E731
    for _ in range(300):
        hq, hkv = rng.choice([(64, 4), (64, 8), (32, 8), (32, 32), (16, 2), (8, 1), (15, 5), (1, 1), (2, 2)])
        topk = rng.randint(1, 256)
        first = rng.randint(0, min(3, topk - 1))
        yield (log(1, 20000), rng.choice([1, 1, 2, 5, 40, 300]), hq, hkv, rng.choice([1, 16, 32, 64, 128, 512]), log(100, 1 << 20), topk, first,
               rng.randint(1, min(3, topk - first)))


def test_a_workspace_of_the_size_that_the_binding_gives_is_enough():
    for T, R, hq, hkv, page, most, topk, first, last in shapes():
        want, at = needed(T, R, hq, hkv, page, most, topk, first, last), (T, R, hq, hkv, page, most)
        size = lambda *choice, **kw: api.vpp_block_select_workspace_size(*at, *choice, **kw)      # noqa: E731
        assert 0 < want == size(topk, first, last), (at, topk, first, last)
        assert size(topk) == max(needed(*at, k, 0, 1) for k in range(1, topk + 1))
        assert want <= min(size(), size(topk), size(topk, first), size(topk, num_last=last)), (at, topk, first, last)


@pytest.mark.parametrize("choice", [(0,), (257,), (8, 9), (8, -1), (8, 0, 0), (8, 4, 5), (256, 256)])
def test_choices_that_the_call_refuses_have_no_size(choice):
    assert api.vpp_block_select_workspace_size(300, 2, 8, 2, 16, 5000, *choice) == 0
