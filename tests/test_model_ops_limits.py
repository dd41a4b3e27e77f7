"""The model operators' limits on sizes, by status code on the host (no launch)."""
import pytest

from paper_2608_05088_gb300 import build, malt, model_ops

A = 1 << 20         # an aligned address that nothing reads


@pytest.fixture(scope="module")
def lib():
    build.build()
    return malt.load()


def test_workspace_of_a_gradient_past_the_limits(lib):
    """0, as for any size that the call refuses."""
    assert lib.malt_embed_workspace_bytes((1 << 30) - 1, 1) > 0 and lib.malt_embed_workspace_bytes(0, 1) > 0
    assert lib.malt_embed_workspace_bytes(1, 1 << 24) > 0
    for tokens, dim in ((1 << 30, 1), (1 << 40, 64), (1, (1 << 24) + 1), (1, 1 << 60)):
        assert lib.malt_embed_workspace_bytes(tokens, dim) == 0
    assert lib.malt_embed_workspace_bytes((1 << 63) - 1, 64) == 0
