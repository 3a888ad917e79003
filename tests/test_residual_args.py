"""Sizes that ResidualAttention refuses before it allocates anything (no GPU needed)."""
import pytest

pytest.importorskip("paper_2607_14898_gb300.flashdec")
from paper_2607_14898_gb300 import ResidualAttention  # noqa: E402


@pytest.mark.parametrize("tokens,width,heads,groups,head_dim", [
    (0, 256, 4, 2, 64), (-8, 256, 4, 2, 64), (12, 256, 4, 2, 64), (16, 0, 4, 2, 64), (16, 264, 4, 2, 64),
    (16, 256, 0, 0, 64), (16, 256, 4, 3, 64), (16, 256, 4, 0, 64), (16, 256, 4, 2, 96)])
def test_sizes(tokens, width, heads, groups, head_dim):
    with pytest.raises(ValueError):
        ResidualAttention(tokens, width, heads, groups, head_dim, None, None, None, None)
