"""Host: the sizes of _projection_forms reach every form that a wide sample of sizes does."""
import numpy as np
import pytest

import _projection_forms as pf
from paper_2609_38386_amd import dlfp as D


@pytest.mark.parametrize("kind", [D.LINEAR_W4, D.GATED_LINEAR_BF16, D.GATED_LINEAR_W4])
def test_every_form_is_among_the_tested_ones(kind):
    """1 to 8191 tokens, 16 to 46000 features, 64 to 32704 columns, workspaces from none to the
    most.  A new choice that reaches other forms fails here and names a size for each."""
    tested = set()
    for size in pf.SIZES[kind]:
        tested |= pf.forms_of(kind, *size)
    rng = np.random.default_rng(kind)
    form, others = D.dlfp_projection_form(), {}
    for i in range(100000):
        m, n, k = (int(2 ** rng.uniform(0, h)) for h in (13, 11.5, 9))
        room = (0, 1 << 20, pf.MOST, pf.MOST)[i % 4]
        for reached in pf.forms_of(kind, m, 16 * n, 64 * k, room, form) - tested:
            others.setdefault(reached, (m, 16 * n, 64 * k, room))
    assert not others
    variants = {f[1] for f in tested if len(f) == 4}
    assert variants == set(range(max(variants) + 1)) - (
        {0, 2, 6} if kind == D.GATED_LINEAR_W4 else set())   # (one block: no gate and up)
