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


def test_norms_of_too_many_heads_are_unsupported(lib):
    """2^33 heads of all tokens are past what a launch counts: a size, not an error of CUDA's."""
    p = model_ops._QK.pack(malt.MALT_F32, malt.MALT_F32, 7, 0, 0, 1e-6, 1, (1 << 31) - 1, 0, 0, 0, 0, A, A, 1, 0, 0)
    many, few = (model_ops._HEADS.pack(A, n, 0, 7 * n, 7) for n in (8, 0))
    assert lib.malt_qk_norm_forward(p, many, few, many, few, None) == malt.MALT_ERR_UNSUPPORTED
    assert lib.malt_qk_norm_forward(p, few, many, few, many, None) == malt.MALT_ERR_UNSUPPORTED
