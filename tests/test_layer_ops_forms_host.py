"""Rows of one leading dimension in one buffer: those that meet are refused before any device is touched (those that lie
between each other's are accepted: test_layer_ops_forms_gpu)."""
import pytest

from paper_2609_11687_amd import kashin as K

X, S = 0x100000, 0x900000
LD = 1100  # rows of 512, so that another 512 fit between them at 512 .. 588


def _norm(t=4, n=512, x=X, r=None, h=None, ldh=LD, y=S, ldy=LD):
    return K.lib().kashin_rmsnorm(t, n, x, 0, LD, r, LD, None, 1e-5, h, ldh, y, 0, ldy, None, 0, None)


@pytest.mark.parametrize("kw", [
    {"y": X + 4 * 511}, {"y": X + 4 * 589}, {"y": X + 4 * LD}, {"y": X + 4 * (2 * LD + 511)}, {"y": X + 4 * (3 * LD - 1)},
    {"y": X - 4 * 511}, {"y": X - 4 * 589}, {"y": X - 4 * LD}, {"y": X - 4 * (LD + 511)},
    {"y": X + 4 * 550, "ldy": LD + 1},                  # another leading dimension: whole ranges count
    {"h": X + 4 * 511}, {"h": X + 4 * LD}, {"h": X + 4 * 550, "ldh": LD - 1}, {"r": X, "h": X + 4},
    {"r": X + 4 * 550, "h": X + 4 * 549}, {"r": X + 4 * 550, "h": X + 4 * (550 + LD)},
    {"t": 1, "y": X + 4 * 511}, {"t": 1, "h": X + 4, "ldh": 512},
])
def test_rows_that_meet_are_refused(kw):
    assert _norm(**kw) == K.KASHIN_E_INVALID
    assert "overlap" in K.lib().kashin_last_error().decode()
