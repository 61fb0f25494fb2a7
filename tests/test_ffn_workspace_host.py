"""Host: the workspace query from Python."""
import pytest

from paper_2609_38386_amd import dlfp as D


@pytest.mark.parametrize("kind", [D.LINEAR_W4, D.GATED_LINEAR_BF16, D.GATED_LINEAR_W4])
@pytest.mark.parametrize("place", range(3))
def test_sizes_past_31_bits_are_refused(kind, place):
    """Of which a C integer would keep the low bits: they are not the workspace of another size."""
    sizes = [256, 2560, 25600]
    assert D.dlfp_projection_workspace(kind, *sizes) > 0
    for far in (1 << 32, 1 << 31, 1 << 40, -1 << 32):
        many = list(sizes)
        many[place] += far
        with pytest.raises(ValueError, match="2\\^31"):
            D.dlfp_projection_workspace(kind, *many)
    assert D.dlfp_projection_workspace(kind, -1, 2560, 25600) == 0
    assert D.dlfp_projection_workspace(kind, 0, 2560, 25600) == 0
    assert D.dlfp_projection_workspace(kind, -1, -16, -64) == 0
