"""Host: the form that a projection takes (dlfp_projection_form_of)."""
import ctypes

import numpy as np
import pytest

from paper_2609_38386_amd import dlfp as D

KINDS = (D.LINEAR_W4, D.GATED_LINEAR_BF16, D.GATED_LINEAR_W4)
MOST = 32 << 20


def _status(kind, m, n, k, room=MOST):
    form = D.dlfp_projection_form()
    return D.lib().dlfp_projection_form_of(kind, m, n, k, room, ctypes.byref(form)), form


def test_the_form_of_some_sizes():
    """Its tile and splits give the bytes of its partial sums, which fit the room and are what the
    workspace query says."""
    rng = np.random.default_rng(11)
    split = 0
    for i in range(6000):
        kind = KINDS[i % 3]
        m, n, k = (int(2 ** rng.uniform(0, h)) for h in (12, 11, 9))
        n, k = 16 * n, 64 * k
        room = int(rng.choice([0, 1 << 16, 1 << 20, MOST]))
        form = D.dlfp_projection_form_of(kind, m, n, k, room)
        assert form.variant >= 0 and 1 <= form.splits <= 8
        rows = form.rows // (1 if kind == D.LINEAR_W4 else 2)
        tiles = -(-m // form.tokens) * -(-n // rows)
        parts = tiles * form.rows * max(16, form.tokens) * 4 * form.splits
        assert form.workspace_bytes == (parts if form.splits > 1 else 0) <= room
        split += form.splits > 1
        if room == MOST:
            assert D.dlfp_projection_workspace(kind, m, n, k) == form.workspace_bytes
    assert split > 300


def test_forms_of_one_size_are_of_one_rule():
    """Weights past the caches: 64 MiB and more, one tile of tokens."""
    for kind, n, k in ((D.LINEAR_W4, 25600, 5120), (D.GATED_LINEAR_W4, 12288, 8192),
                       (D.GATED_LINEAR_BF16, 12288, 4096)):
        assert D.dlfp_projection_form_of(kind, 2, n, k, MOST).past_caches == 1
        assert D.dlfp_projection_form_of(kind, 2, n // 16, k, MOST).past_caches == 0
        assert D.dlfp_projection_form_of(kind, 4096, n, k, MOST).past_caches == 0


@pytest.mark.parametrize("kind,m,n,k", [
    (D.GATED_LINEAR_W4, 1, 1 << 28, 128), (D.LINEAR_W4, 1, 1 << 29, 128),
    (D.LINEAR_W4, 1 << 30, 16, 64), (D.GATED_LINEAR_W4, 1 << 30, 16, 64),
    (D.GATED_LINEAR_BF16, 1 << 30, 16, 64), (D.GATED_LINEAR_BF16, 1, 1 << 28, 64),
    (D.GATED_LINEAR_W4, 3, (1 << 29) + 16, 64), (D.LINEAR_W4, 1, (1 << 30) - 16, 64)])
def test_sizes_that_some_form_can_launch_are_taken(kind, m, n, k):
    """2^32 threads and more in one form leave the others."""
    status, form = _status(kind, m, n, k)
    assert status == 0 and form.variant >= 0
    rows = form.rows // (1 if kind == D.LINEAR_W4 else 2)
    # (at least 64 threads to a tile, at most 512)
    assert -(-m // form.tokens) * -(-n // rows) * form.splits * 64 < 1 << 32


def test_every_size_below_the_documented_limit_is_taken():
    """512 threads for each 256 tokens and 256 features (gated: 128) below 2^32."""
    rng = np.random.default_rng(2)
    taken = 0
    for i in range(4000):
        kind = KINDS[i % 3]
        m = int(2 ** rng.uniform(0, 31))
        n = 16 * int(2 ** rng.uniform(0, 27))
        k = 64 * int(2 ** rng.uniform(0, 8))
        features = 256 if kind == D.LINEAR_W4 else 128
        widest = -(-m // 256) * -(-n // features) * 512
        status, _ = _status(kind, m, n, k)
        if widest < 1 << 32 and max(m, n) <= (1 << 31) - 1025:
            assert status == 0
            taken += 1
        else:
            assert status in (0, -2)
    assert taken > 1000


@pytest.mark.parametrize("args,status", [
    ((3, 1, 16, 64), -1), ((-1, 1, 16, 64), -1), ((0, 0, 16, 64), -1), ((0, 1, 0, 64), -1),
    ((0, 1, 16, -64), -1), ((0, 1, 24, 64), -5), ((1, 1, 16, 96), -5), ((2, 1, 16, 1 << 22), -2),
    ((0, 1 << 30, 1 << 30, 64), -2), ((0, (1 << 31) - 1, 16, 64), -2)])
def test_refusals(args, status):
    """A refused form stays as it was."""
    form = D.dlfp_projection_form(variant=-7)
    assert D.lib().dlfp_projection_form_of(*args, MOST, ctypes.byref(form)) == status
    assert form.variant == -7
    with pytest.raises(D.DlfpError):
        D.dlfp_projection_form_of(*args, MOST)
    assert D.lib().dlfp_projection_form_of(0, 1, 16, 64, MOST, None) == -1


def test_sizes_past_31_bits_are_refused_from_python():
    for sizes in (((1 << 32) + 1, 16, 64), (1, (1 << 32) + 16, 64), (1, 16, (1 << 32) + 64)):
        with pytest.raises(ValueError, match="2\\^31"):
            D.dlfp_projection_form_of(D.LINEAR_W4, *sizes, MOST)
