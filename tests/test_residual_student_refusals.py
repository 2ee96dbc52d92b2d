"""Residual blocks and heads that a token student cannot have (no GPU)."""
import pytest

from paper_2509_26092_amd import distill


@pytest.mark.parametrize("kw", [dict(blocks=-1), dict(blocks=-1, dropout=0.1), dict(blocks=1, heads=0),
                                dict(blocks=2, heads=-8)])
def test_numbers_of_blocks_and_heads(kw):
    """Fewer than no blocks were taken for none, with a dropout that nothing took."""
    with pytest.raises(ValueError, match="residual blocks"):
        distill.TokenStudent(20, **kw)
