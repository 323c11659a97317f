"""The layer operators' further forms on the GPU against float64: every vector length, every tile of the products whole and by
expert, rows that no expert has, values that are not finite, matrices of uneven magnitude, rows side by side in one
buffer.  Tolerances as in test_layer_ops_gpu, whose helpers these tests use; where one differs its derivation stands
beside it."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import test_layer_ops_gpu as base
from paper_2609_11687_amd import kashin as K
from test_layer_ops_gpu import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    K.lib()


# ----------------------------------------------------------------------------- norm
@pytest.mark.parametrize("n", [300, 1024, 5000, 12000])
@pytest.mark.parametrize("group", [0, 32, 128])
def test_rmsnorm_groups_with_an_infinite_y(n, group):
    """A group of 8-bit entries with an infinite one is a group that has no scale: scale NaN and zeros, as with a NaN."""
    rng = np.random.default_rng(n + group)
    x = torch.from_numpy(rng.standard_normal((6, n)).astype(np.float32)).cuda()
    x[:, 5], x[:, 70] = 1.5, -1.5
    x[4] *= 1e-25  # the squares underflow
    x[5] = 0.0
    w = torch.ones(n, device="cuda")
    w[5], w[70] = math.inf, 3e38  # at 70 the product passes the largest float
    cols = -(-n // group) if group else 1
    for weight, eps in ((w, 1e-6), (None, 0.0)):
        y = torch.empty((6, n), device="cuda")
        q, s = torch.full((6, n), 7.0).to(torch.float8_e4m3fn).cuda(), torch.full((6, cols), 7.0, device="cuda")
        K.kashin_rmsnorm(x, None, weight, eps, None, y)
        K.kashin_rmsnorm(x, None, weight, eps, None, q, s, group)
        torch.cuda.synchronize()
        y, q, s = base._f64(y), base._f64(q), base._f64(s)
        for g in range(cols):
            part = slice(g * group, (g + 1) * group) if group else slice(0, n)
            lost = ~np.isfinite(y[:, part]).all(1)
            assert (q[lost][:, part] == 0).all() and np.isnan(s[lost, g]).all(), (g, q[lost][:, part], s[lost, g])
            kept = y[~lost][:, part]
            assert np.allclose(s[~lost, g], np.abs(kept).max(1, initial=0.0) / 448, rtol=2.0 ** -22, atol=0)
            if eps == 0.0:
                assert lost[4] and lost[5]
            elif g == 0:
                assert lost[:4].all()


@pytest.mark.parametrize("n,t", [(8, (1 << 22) + 7), (520, (1 << 20) + 5), (2050, (1 << 20) + 1)])
def test_rmsnorm_of_more_rows_than_a_grid_holds(n, t):
    """Workgroups that walk several rows: as calls on parts of the rows, bit for bit."""
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.empty((t, n), dtype=torch.bfloat16, device="cuda")
    for part in x.split(1 << 18):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda"))
    q, s = torch.empty((t, n), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((t, 1), device="cuda")
    K.kashin_rmsnorm(x, None, None, 1e-6, None, q, s)
    for i in range(0, t, 1 << 18):
        part = x[i:i + (1 << 18)]
        q1, s1 = torch.empty_like(q[i:i + (1 << 18)]), torch.empty_like(s[i:i + (1 << 18)])
        K.kashin_rmsnorm(part, None, None, 1e-6, None, q1, s1)
        assert torch.equal(q1.view(torch.uint8), q[i:i + (1 << 18)].view(torch.uint8)) and torch.equal(s1, s[i:i + (1 << 18)])


# ----------------------------------------------------------------------------- lengths
@pytest.mark.parametrize("back", [False, True])
def test_products_of_every_compiled_length(back):
    for n in (n for n in range(2, 20000, 2) if K.kashin_supported_n(n)):
        print(f"product n={n} back={back}", flush=True)
        case = Case(n, 37)
        for t, dtype, out, xg in ((1, "e4m3", "f32", 64), (2, "f32", "f32", 0), (5, "f16", "f16", 0), (19, "e4m3", "bf16", 0),
                                  (70, "bf16", "f32", 0)):
            x, y = base._product(case, t, dtype, out, back, xg)
            base._check(case, y, x, out, back)


# ----------------------------------------------------------------------------- tiles
@pytest.mark.parametrize("n,m,t", [(96, 1000, 130), (172, 1000, 130), (512, 1000, 130),  # 32 x 32
                                   (96, 1000, 400), (172, 1000, 400), (512, 1000, 400),  # 32 x 64
                                   (96, 8200, 100), (172, 8200, 250)])                   # 256 x 64, 256 x 128
def test_products_of_every_tile(n, m, t):
    print(f"product n={n} m={m} t={t}", flush=True)
    case = Case(n, m)
    for dtype, out in (("bf16", "bf16"), ("f16", "f16"), ("e4m3", "f32")):
        x, y = base._product(case, t, dtype, out, False, 32 if dtype == "e4m3" else 0)
        base._check(case, y, x, out, False)


@pytest.mark.parametrize("n,groups,t", [(64, 128, 300), (64, 64, 1601)])
def test_products_of_16_bit_rows_of_many_groups(n, groups, t):
    """Rows whose P x passes through memory."""
    case = Case(n, 5, groups)
    for dtype, out in (("f16", "f32"), ("f16", "bf16"), ("bf16", "f16")):
        x, y = base._product(case, t, dtype, out, False)
        base._check(case, y, x, out, False)


def _ragged(experts, each, seed):
    """Row counts of `experts` experts, `each` on average, from none to three times that."""
    rng = np.random.default_rng(seed)
    share = rng.uniform(0.0, 3.0, experts) ** 2
    share[experts // 2] = 0.0
    return list(rng.multinomial(experts * each, share / share.sum()))


def _grouped(case, counts, first, spare, dtype, out, back, seed=0):
    """Products by expert, the rows outside the offsets' range holding NaN and infinities (scales too), against float64."""
    rng = np.random.default_rng([seed, len(counts)])
    used = int(sum(counts))
    t = first + used + spare
    wx, wy = (case.m, case.k) if back else (case.k, case.m)
    x = base._rows(rng, t, wx, dtype)
    scales = None
    if dtype == "e4m3":
        scales = torch.from_numpy(rng.uniform(0.1, 2.0, (t, 1)).astype(np.float32)).cuda()
    x64 = base._f64(x) * (base._f64(scales) if scales is not None else 1.0)
    for row in list(range(first)) + list(range(first + used, t)):
        x[row] = math.nan
        if dtype != "e4m3":
            x[row, ::3] = math.inf
            x[row, 1::3] = -math.inf
        else:
            scales[row] = math.inf if row % 2 else math.nan
    off = first + np.concatenate([[0], np.cumsum(counts)])
    flat, y = base._buffer(t, wy, out)
    K.kashin_matmul_experts(case.plan, *case.dev, torch.from_numpy(off.astype(np.int64)).cuda(), x, y, case.work(t, back), back,
                            scales, 0, rot_seed=case.rot)
    torch.cuda.synchronize()
    for e in range(case.experts):
        base._check(case, y[off[e]:off[e + 1]], x64[off[e]:off[e + 1]], out, back, e)
    f = flat.to(torch.float32)
    assert (f[:first * wy] == 7).all() and (f[(first + used) * wy:] == 7).all()


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("n,groups,m,experts,each", [
    (256, 2, 35, 5, 3), (96, 1, 70, 3, 12),
    (256, 1, 1000, 8, 20), (96, 1, 1000, 8, 20),    # 32 x 32
    (256, 1, 1200, 6, 45), (172, 1, 1200, 6, 45),   # 32 x 64
    (64, 1, 1800, 32, 30), (256, 1, 300, 32, 130), (172, 1, 300, 32, 130),  # 256 x 64
    (256, 1, 4100, 5, 250)])                        # 256 x 128
def test_experts_of_every_tile(n, groups, m, experts, each, back):
    print(f"experts {experts} of {each} n={n} m={m} back={back}", flush=True)
    case = Case(n, m, groups, experts=experts)
    counts = _ragged(experts, each, m)
    for dtype, out in (("bf16", "bf16"), ("f32", "f32"), ("e4m3", "bf16")):
        _grouped(case, counts, 3, 2, dtype, out, back)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("n,groups,rot", [(512, 1, 3), (64, 3, 7)])
def test_experts_of_rotated_weights_beside_rows_of_nobody(n, groups, rot, back):
    for each in (4, 40):
        case = Case(n, 90, groups, experts=4, rot=rot)
        for dtype, out in (("f16", "f32"), ("e4m3", "bf16")):
            _grouped(case, _ragged(4, each, n), 1, 3, dtype, out, back)


# ----------------------------------------------------------------------------- magnitudes
@pytest.mark.parametrize("t", [1, 9, 15, 16, 40, 70, 130])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_transposed_groups_of_uneven_magnitude(t, out):
    """The columns of a group come from its own centres: those scaled by a power of two scale the columns, bit for bit,
    whatever the other groups hold; the same for a factor (where the other one is zero)."""
    case = Case(256, 300, 3)
    cu, cv, ce = case.dev
    x = base._rows(np.random.default_rng(t), t, case.m, "f32")

    def product(centers):
        y = torch.empty((t, case.k), dtype=base.DT[out], device="cuda")
        K.kashin_matmul_t(case.plan, cu, cv, centers, x, y, case.work(t, True))
        return y.to(torch.float32).view(t, 3, 256)

    y = product(ce)
    by = torch.tensor([2.0 ** -30, 1.0, 2.0 ** -45], device="cuda")
    assert torch.equal(product((ce.view(300, 3, 8) * by[:, None]).view(-1, 2, 4)), y * by[:, None])
    for f in (0, 1):
        one = ce.clone().view(300, 3, 2, 4)
        one[:, :, 1 - f] = 0.0
        one[:, 0, 1 - f] = 2.0 ** -6
        y = product(one.view(-1, 2, 4))
        other = one.clone()
        other[:, 0, 1 - f] = 1.0  # group 0's other factor far above
        other[:, 1:] *= 2.0 ** -40
        assert torch.equal(product(other.view(-1, 2, 4))[:, 1:], y[:, 1:] * 2.0 ** -40)


@pytest.mark.parametrize("t", [3, 12, 20, 70, 130])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("factor", [0, 1])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_products_with_one_centre_that_is_not_finite(t, out, factor, value):
    """One centre of a row of W_hat: its column is NaN, transposed the columns of its group, whichever entries take that
    centre, and nothing else."""
    case = Case(256, 40, 2)
    cu, cv, ce = case.dev
    ce = ce.clone()
    ce[7 * 2 + 1, factor, 2] = value
    x = base._rows(np.random.default_rng(0), t, case.k, "f32")
    y = torch.empty((t, 40), dtype=base.DT[out], device="cuda")
    K.kashin_matmul(case.plan, cu, cv, ce, x, y, case.work(t, False))
    assert y[:, 7].isnan().all()
    assert y[:, [i for i in range(40) if i != 7]].isfinite().all()
    x = base._rows(np.random.default_rng(0), t, 40, "f32")
    x[0] = 0.0
    y = torch.empty((t, 512), dtype=base.DT[out], device="cuda")
    K.kashin_matmul_t(case.plan, cu, cv, ce, x, y, case.work(t, True))
    assert y[:, 256:].isnan().all() and y[:, :256].isfinite().all()


@pytest.mark.parametrize("t", [1, 3, 7])
@pytest.mark.parametrize("n,groups,m", [(512, 1, 200), (256, 3, 1000), (4096, 1, 700)])
def test_transposed_bf16_results_of_few_rows(n, groups, m, t):
    """Few rows cost no more with operands of two parts, so nearly every bf16 result is the exact one's rounding.  An fp32
    result is off by 1e-6 of a typical one at most (NORM).  An entry then rounds elsewhere where a border between two
    bf16 numbers (2^-8 to 2^-7 of |y| apart) lies within that: 2 * 1e-6 * 2^8 = 5e-4 for a typical entry, about five times
    that on average over normally distributed ones (smaller entries have closer borders).  1 in 100 is allowed."""
    case = Case(n, m, groups)
    for dtype in ("bf16", "f32", "e4m3"):
        x, got = base._product(case, t, dtype, "bf16", True, 64 if dtype == "e4m3" else 0)
        base._check(case, got, x, "bf16", True)
        want = torch.from_numpy(x @ case.w[0]).to(torch.bfloat16)
        assert (got.cpu() != want).float().mean() <= 0.01, (dtype, (got.cpu() != want).float().mean())


# ----------------------------------------------------------------------------- rows side by side
def test_rows_side_by_side_in_one_buffer():
    """Column ranges of one buffer are rows of the same leading dimension that lie between each other's and do not overlap."""
    t, n, m = 9, 512, 100
    rng = np.random.default_rng(0)
    wide = torch.full((t, 4 * n + 64), 7.0, device="cuda")
    x, r, h, y = (wide[:, i * n:(i + 1) * n] for i in range(4))
    s = wide[:, 4 * n:]
    a, b = (torch.from_numpy(rng.standard_normal((t, n)).astype(np.float32)).cuda() for _ in range(2))
    x.copy_(a)
    r.copy_(b)
    h1, y1 = torch.empty_like(a), torch.empty_like(a)
    K.kashin_rmsnorm(a, b, None, 1e-5, h1, y1)
    K.kashin_rmsnorm(x, r, None, 1e-5, h, y)
    torch.cuda.synchronize()
    assert torch.equal(h, h1) and torch.equal(y, y1) and torch.equal(x, a) and torch.equal(r, b) and (s == 7).all()
    case = Case(n, m)
    for back in (False, True):
        wx, wy = (m, n) if back else (n, m)
        f = K.kashin_matmul_t if back else K.kashin_matmul
        for dtype in ("f32", "f16"):
            rows = base._rows(rng, t, wx, dtype)
            z1 = torch.empty((t, wy), dtype=base.DT[dtype], device="cuda")
            f(case.plan, *case.dev, rows, z1, case.work(t, back))
            both = torch.full((t, wx + wy + 3), 7.0, dtype=base.DT[dtype], device="cuda")
            for at_x, at_z in ((0, wx + 3), (wy + 1, 0)):
                both.fill_(7.0)
                u, z = both[:, at_x:at_x + wx], both[:, at_z:at_z + wy]
                u.copy_(rows)
                f(case.plan, *case.dev, u, z, case.work(t, back))
                torch.cuda.synchronize()
                assert torch.equal(z, z1) and torch.equal(u, rows)
                rest = torch.ones(wx + wy + 3, dtype=torch.bool, device="cuda")
                rest[at_x:at_x + wx] = False
                rest[at_z:at_z + wy] = False
                assert (both[:, rest] == 7).all()
    # rows that do meet, in one buffer with one leading dimension
    flat = torch.empty(t * 2 * n + n, device="cuda")
    x = flat[:t * 2 * n].view(t, 2 * n)[:, :n]
    for at in (n - 1, 2 * n - m + 1, 2 * n, 0):
        y = flat[at:at + (t - 1) * 2 * n].view(t - 1, 2 * n)[:, :m]
        with pytest.raises(K.KashinError, match="overlap"):
            K.kashin_matmul(case.plan, *case.dev, x[:t - 1], y, case.work(t, False))


# ----------------------------------------------------------------------------- the largest sizes
def test_products_of_the_most_matrix_rows():
    """2^24 matrix rows, 4.3 GB of codes a factor: as the products of parts of the matrix.  Transposed, a sum of 2^24 terms:
    a split's chain of up to 1024 steps of 7 additions and at most 512 splits, 2^-24 (sqrt(7168 / 6) + sqrt(512 / 6)) =
    2.6e-6 of a typical result; the parts' own sums are shorter.  Four times that is allowed."""
    n, m, t = 1024, 1 << 24, 2
    plan = K.kashin_plan(n, 3, 1)
    g = torch.Generator(device="cuda").manual_seed(0)
    cu, cv = torch.empty((2, m, n // 4), dtype=torch.uint8, device="cuda")
    for c in (cu, cv):
        for part in c.split(1 << 20):
            part.random_(0, 256, generator=g)
    ce = (torch.randn((m, 2, 4), generator=g, device="cuda") * 0.02).sort(-1).values

    def run(f, x, lo, hi, width):
        y = torch.empty((t, width), device="cuda")
        back = f is K.kashin_matmul_t
        work = torch.empty(K.kashin_matmul_workspace_bytes(n, hi - lo, 1, t, 1, back), dtype=torch.uint8, device="cuda")
        f(plan, cu[lo:hi], cv[lo:hi], ce[lo:hi], x, y, work)
        return y
    x = torch.randn((t, n), generator=g, device="cuda")
    y = run(K.kashin_matmul, x, 0, m, m)
    for lo in (0, (1 << 23) - 256, m - 512):
        assert torch.equal(y[:, lo:lo + 512], run(K.kashin_matmul, x, lo, lo + 512, 512)), lo
    x = torch.randn((t, m), generator=g, device="cuda")
    y = run(K.kashin_matmul_t, x, 0, m, n).double()
    step = 1 << 20
    want = sum(run(K.kashin_matmul_t, x[:, lo:lo + step], lo, lo + step, n).double() for lo in range(0, m, step))
    assert (y - want).norm() <= 4 * 2.6e-6 * want.norm()


@pytest.mark.parametrize("back", [False, True])
def test_products_of_the_most_rows(back):
    case = Case(64, 70)
    t = 1 << 16
    for dtype, out in (("bf16", "bf16"), ("f16", "f32")):
        x, y = base._product(case, t, dtype, out, back)
        for part in (slice(0, 300), slice(t // 2 - 100, t // 2 + 100), slice(t - 300, t)):
            base._check(case, y[part], x[part], out, back)


@pytest.mark.parametrize("back", [False, True])
def test_products_of_the_longest_rows(back):
    case = Case(16384, 20, 64)
    for t, dtype, out in ((2, "f32", "f32"), (20, "bf16", "f32")):
        x, y = base._product(case, t, dtype, out, back)
        base._check(case, y, x, out, back)


@pytest.mark.parametrize("back", [False, True])
def test_the_most_experts(back):
    case = Case(64, 16, 2, experts=1024)
    for each in (1, 30):
        _grouped(case, _ragged(1024, each, each), 2, 1, "bf16", "f32", back)


# ----------------------------------------------------------------------------- graphs
def test_captured_rotated_products_replay():
    """Rotated products in tiles and by expert with bf16 results in one captured graph: every replay as the eager calls, bit for
    bit, with eager work on other inputs in between."""
    case, ex = Case(512, 700, rot=4), Case(256, 130, 2, experts=3, rot=9)
    t = 200
    rng = np.random.default_rng(0)
    off = torch.tensor([1, 90, 90, 190], device="cuda")

    def state():
        z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        return {"x": z(t, 512), "y": z(t, 700), "z": z(t, 512), "e": z(t, 130), "et": z(t, 512),
                "work": [case.work(t, False), case.work(t, True), ex.work(t, False), ex.work(t, True)]}

    def step(s):
        K.kashin_matmul(case.plan, *case.dev, s["x"], s["y"], s["work"][0], rot_seed=case.rot)
        K.kashin_matmul_t(case.plan, *case.dev, s["y"], s["z"], s["work"][1], rot_seed=case.rot)
        K.kashin_matmul_experts(ex.plan, *ex.dev, off, s["z"], s["e"], s["work"][2], rot_seed=ex.rot)
        K.kashin_matmul_experts(ex.plan, *ex.dev, off, s["e"], s["et"], s["work"][3], True, rot_seed=ex.rot)

    s, eager = state(), state()
    step(eager)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(s)
    for i in range(4):
        x = base._rows(rng, t, 512, "bf16")
        s["x"].copy_(x)
        eager["x"].copy_(x)
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        for key in ("y", "z", "e", "et"):
            assert s[key].isfinite().all() and torch.equal(s[key].view(torch.uint8), eager[key].view(torch.uint8)), (i, key)
