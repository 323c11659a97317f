"""Host-side checks of the layer operators.  Rows of one leading dimension in one buffer: those that meet are refused before
any device is touched (those that lie between each other's are accepted: test_layer_ops_forms_gpu).  Workspaces."""
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


def test_workspace_holds_p_of_x_only_where_it_passes_through_memory():
    """Two parts of two factors, a row's exponent and one fp32 copy of x, and P x besides for rows of very many groups; never
    less for more rows."""
    size = K.kashin_matmul_workspace_bytes
    up = lambda v: -(-v // 256) * 256  # noqa: E731
    for n, groups, rows in ((4096, 1, (1, 100, 65536)), (256, 16, (1, 4096)), (64, 128, (1, 256, 257, 60000))):
        k = n * groups
        chunks = -(-groups * -(-n // 64) // 4) * 4
        for t in rows:
            copies = 1 if groups == 1 or t * groups * k <= 2 ** 28 else 2
            assert size(n, 1000, groups, t) == copies * up(4 * t * k) + up(4 * t) + 4 * chunks * 8 * t * 16
    sizes = [size(64, 1000, 128, t) for t in range(600)]
    assert sizes == sorted(sizes)
