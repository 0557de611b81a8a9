"""Workspaces of the shared-prefix attention (no GPU needed)."""
import pytest

from paper_2609_36938_b200 import binding as B
from paper_2609_36938_b200 import build


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return B.load()


def latent(n, page, prefix, most):
    return B.attn_decode_shared_workspace_size(n, 128, 576, 1, 512, page, prefix, most)


def test_latent_workspace_is_bounded():
    """A piece's table holds its own pages, and no more than 8192 pieces are made at a time: 2 GB of outputs, 128 MB of tokens, and the tables."""
    for n in (64, 300, 1024, 8000):
        for page in (1, 16, 64):
            assert latent(n, page, 0, 131072) <= (1 << 31) + 8192 * 4 * (2 * 4096 + 200) + 8 * n * 131072, (n, page)
    # pages of one token: not more than twice what pages of 64 take
    assert latent(64, 1, 0, 131072) <= 2 * latent(64, 64, 0, 131072)


def test_latent_workspace_covers_both_kernels():
    """Values that are no part of the keys go by the general kernel, whose lists hold every session's tokens and pages."""
    for n, page, prefix, most in ((1, 64, 0, 1), (1024, 64, 0, 131072), (8000, 1, 100, 9000), (3, 16, 70, 300)):
        pages = -(-prefix // page) + -(-most // page) - prefix // page
        assert latent(n, page, prefix, most) >= n * (4 * most + 4 * pages + 8)
