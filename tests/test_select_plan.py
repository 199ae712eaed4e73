"""The host's plan of vpp_block_select, without a GPU: what its workspace has room for."""
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
    size = lambda T: api.vpp_block_select_workspace_size(T, 1, 32, 32, 64, 131072, topk=128)      # noqa: E731
    assert size(256 + rest) >= size(256 + 5) + 4 * 32 * 4
    assert size(512 + rest + 5) == size(512 + 256)
