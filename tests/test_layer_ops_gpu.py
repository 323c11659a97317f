"""The operators of a quantised model's layers on the GPU against float64: the norm with its 8-bit output, the
products from the codes, transposed and grouped by expert, and a run of them together.

Tolerances, derived before the first run.  A product's error in fp32 has three parts: P x (each transform's
stages, 2^-22 of the row's norm at most on average), the operands (two fp16 parts each, 2^-21 of a term) and the
sums.  With independent roundings their quadratic sum stays under 5e-7 of the result's norm over these sizes; twice that
is allowed (NORM).  An entry is off by at most 2^-24 (L + 64) of the sum of its terms' magnitudes, L the longest chain of
additions (here: K / 32, or m).  The output's rounding adds half a step, finfo.eps / 2.  bf16 results of the
product with the matrix's rows come from operands rounded to fp16: two roundings of 2^-11 a term."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import oracle.kashin_ref as ref
from paper_2609_11687_amd import kashin as K
from paper_2609_11687_amd import optq

pytestmark = pytest.mark.gpu

NORM = 1e-6
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}  # half the smallest step


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    K.lib()


def _f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _rows(rng, t, n, dtype, ld=None, shift=0):
    """t rows of n activations of `dtype` on the GPU with leading dimension `ld`, the first `shift` entries into a buffer."""
    ld = ld or n
    x = rng.standard_normal((t, n))
    x[:, rng.integers(0, n, max(1, n // 200))] *= 20.0
    flat = torch.full((shift + t * ld + 8,), 3.0).to(DT[dtype]).cuda()
    v = flat[shift:shift + t * ld].view(t, ld)[:, :n]
    v.copy_(torch.from_numpy(x).cuda().to(DT[dtype]))
    return v


def _buffer(t, n, dtype, ld=None, shift=0, fill=7.0):
    ld = ld or n
    flat = torch.full((shift + t * ld + 8,), fill).to(DT[dtype]).cuda()
    return flat, flat[shift:shift + t * ld].view(t, ld)[:, :n]


# ----------------------------------------------------------------------------- norm
def _norm64(x, r, w, eps):
    s = x + (r if r is not None else 0.0)
    y = s / np.sqrt((s * s).mean(1, keepdims=True) + eps)
    return s, y * (w if w is not None else 1.0)


# of a value: the sum of squares (in a thread 8 or 16 terms, then at most 10 levels), its root, two products
NORM_REL = 2.0 ** -24 * 32


@pytest.mark.parametrize("n", [1, 7, 8, 33, 64, 500, 512, 513, 2048, 2055, 4096, 4099, 8192, 8200, 16383, 16384])
@pytest.mark.parametrize("dtype,out,group", [("f32", "f32", 0), ("f16", "e4m3", 0), ("bf16", "e4m3", 128),
                                             ("bf16", "bf16", 0), ("f32", "e4m3", 32), ("f16", "f16", 0),
                                             ("bf16", "e4m3", 256), ("f16", "e4m3", 64)])
def test_rmsnorm_matches_float64(n, dtype, out, group):
    print(f"rmsnorm n={n} {dtype} -> {out} group {group}", flush=True)
    rng = np.random.default_rng(n + group)
    for t, ld, shift, residual, weight in ((1, n, 0, True, True), (5, n + 3, 1, True, False), (9, n, 0, False, True)):
        x = _rows(rng, t, n, dtype, ld, shift)
        r = _rows(rng, t, n, dtype, ld, 2 * shift) if residual else None
        w = _rows(rng, 1, n, dtype)[0] if weight else None
        hflat, h = _buffer(t, n, dtype, n + 5, shift)
        yflat, y = _buffer(t, n, out, n + 1, shift)
        s = torch.full((t, -(-n // group) if group else 1), 7.0, device="cuda") if out == "e4m3" else None
        K.kashin_rmsnorm(x, r, w, 1e-5, h, y, s, group)
        torch.cuda.synchronize()
        sum64, y64 = _norm64(_f64(x), None if r is None else _f64(r), None if w is None else _f64(w), 1e-5)
        assert (np.abs(_f64(h) - sum64) <= HALF_STEP[dtype] * np.abs(sum64) * (1 + 1e-6) + LEAST[dtype]).all()
        if out == "e4m3":
            for g in range(s.shape[1]):
                part = slice(g * group, (g + 1) * group) if group else slice(0, n)
                top = np.abs(y64[:, part]).max(1)
                assert np.allclose(_f64(s)[:, g], top / 448, rtol=NORM_REL + 2.0 ** -24, atol=0)
                v = y64[:, part] / _f64(s)[:, g:g + 1]
                off = np.abs(_f64(y)[:, part] - v)
                assert (off <= 2.0 ** -4 * np.abs(v) * (1 + 1e-4) + 2.0 ** -10 * (1 + 1e-4)).all()
        else:
            assert (np.abs(_f64(y) - y64) <= (HALF_STEP[out] + NORM_REL) * np.abs(y64) + LEAST[out]).all()
        # nothing outside the rows
        for flat, v, wide in ((hflat, h, n + 5), (yflat, y, n + 1)):
            f = flat.to(torch.float32)
            assert (f[:shift] == 7).all() and (f[shift + t * wide:] == 7).all()
            assert (f[shift:shift + t * wide].view(t, wide)[:, n:] == 7).all()


def test_rmsnorm_in_place_many_rows_repeats():
    rng = np.random.default_rng(3)
    for n, t in ((64, 4097), (768, 1500), (5000, 700)):
        x, r = _rows(rng, t, n, "bf16"), _rows(rng, t, n, "bf16")
        y = torch.empty_like(x)
        h = torch.empty_like(x)
        K.kashin_rmsnorm(x, r, None, 1e-6, h, y)
        y2, r2, x2 = torch.empty_like(x), r.clone(), x.clone()
        K.kashin_rmsnorm(x, r2, None, 1e-6, r2, y2)
        y3 = torch.empty_like(x)
        K.kashin_rmsnorm(x2, r, None, 1e-6, x2, y3)
        one = torch.empty_like(x[:1])
        K.kashin_rmsnorm(x[t - 1:], r[t - 1:], None, 1e-6, None, one)
        torch.cuda.synchronize()
        for a, b in ((h, r2), (h, x2), (y, y2), (y, y3), (y[t - 1:], one)):
            assert torch.equal(a, b)


def test_rmsnorm_zeros_and_values_that_are_not_finite():
    n = 300
    x = torch.ones((6, n), device="cuda")
    x[1] = 0.0
    x[2, 40] = math.nan
    x[3, 299] = math.inf
    x[4] = 1e20  # the sum of squares passes the largest float
    x[5] = 1e-30
    y, h = torch.empty_like(x), torch.empty_like(x)
    K.kashin_rmsnorm(x, None, None, 0.0, h, y)
    q, s = torch.empty((6, n), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((6, 3), device="cuda")
    K.kashin_rmsnorm(x, None, None, 1e-6, None, q, s, 128)
    torch.cuda.synchronize()
    assert torch.equal(h.view(torch.int32), x.view(torch.int32))
    y, q, s = y.cpu(), q.to(torch.float32).cpu(), s.cpu()
    assert torch.allclose(y[0], torch.ones(n), rtol=1e-6) and y[1].isnan().all() and y[2].isnan().all()
    assert y[3, 299].isnan() and (y[3, :299] == 0).all() and (y[4] == 0).all()
    assert (q[1] == 0).all() and (s[1] == 0).all()
    assert (q[2] == 0).all() and s[2].isnan().all()
    assert (q[3] == 0).all() and (s[3, :2] == 0).all() and s[3, 2].isnan()
    assert (q[4] == 0).all() and (s[4] == 0).all()
    assert (q[0] == 448).all() and (q[5] == 448).all()


# ----------------------------------------------------------------------------- products
class Case:
    """Codes with centres on the GPU, W_hat and its factors' magnitudes in float64."""

    def __init__(self, n, m, groups=1, experts=1, seed=0, rot=None):
        rng = np.random.default_rng([n, m, groups, experts, seed])
        rows, nb = experts * m * groups, n // 4
        cu, cv = (rng.integers(0, 256, (rows, nb), dtype=np.uint8) for _ in range(2))
        ce = np.sort(rng.standard_normal((rows, 2, 4)) * [[[0.02], [0.006]]], axis=2) * rng.uniform(0.2, 3.0, (rows, 1, 1))
        ce = ce.astype(np.float32)
        self.n, self.m, self.groups, self.experts, self.rot, self.k = n, m, groups, experts, rot, n * groups
        self.seed = seed + 17
        self.plan = K.kashin_plan(n, self.seed, 1)
        self.dev = tuple(torch.from_numpy(a).cuda() for a in (cu, cv, ce))
        self.eps = ref.sign_mask(n, self.seed)
        ce64 = ce.astype(np.float64)
        u, v = (np.take_along_axis(ce64[:, f], ref.unpack2bit(c, n).astype(np.int64), 1) for f, c in ((0, cu), (1, cv)))
        w = u + ref.apply_p(v, self.eps)
        if rot is not None:
            w = ref.rotate(w, rot, inverse=True)
        self.u, self.v, self.w = (a.reshape(experts, m, self.k) for a in (u, v, w))
        top = np.abs(ce64).max(2)  # of each row's centres, over its entries
        self.top = [np.broadcast_to(top[:, f, None], u.shape).reshape(experts, m, self.k) for f in (0, 1)]

    def px(self, x):
        """R x and P R x of rows of k."""
        g = x.reshape(-1, self.n)
        g = ref.rotate(g, self.rot) if self.rot is not None else g
        return g.reshape(x.shape), ref.apply_p(g, self.eps).reshape(x.shape)

    def work(self, t, back):
        return torch.empty(K.kashin_matmul_workspace_bytes(self.n, self.m, self.groups, t, self.experts, back),
                           dtype=torch.uint8, device="cuda")


def _check(case, got, x, out, back, e=0):
    """got (device rows) against float64 for one expert's rows x (numpy)."""
    if not x.shape[0]:
        return
    t = x.shape[0]
    w, u, v = case.w[e], case.u[e], case.v[e]
    want = x @ w if back else x @ w.T
    if back:
        zu, zv = np.abs(x) @ np.abs(u), np.abs(x) @ np.abs(v)
        # P and the rotation spread a group's errors over its entries
        def spread(z):
            g = z.reshape(t, case.groups, case.n)
            return np.broadcast_to(np.sqrt((g * g).sum(2, keepdims=True)), g.shape).reshape(z.shape)
        mag = spread(zu) + spread(zv) if case.rot is not None else zu + spread(zv)
        chain = case.m
    else:
        xr, xp = case.px(x)
        mag = np.abs(xr) @ np.abs(u).T + np.abs(xp) @ np.abs(v).T
        # P's error reaches every entry of P x
        mag = mag + np.linalg.norm(x, axis=1)[:, None] * np.linalg.norm(v, axis=1)[None, :]
        chain = case.k / 32
    term = 2.0 ** -24 * (chain + 64)
    norm = NORM
    room = 1.01 * term * mag
    if out == "bf16" and not back:
        room = room + 2 * 2.0 ** -11 * mag
        norm += 2.0 ** -11
    elif out == "bf16":
        # x times a row's four coefficients is rounded to fp16: with centres up to q they are at most q, 6 q, 5 q and
        # 4 q, and meet functions of the code up to 1, 1, 2 and 4: 33 q in all; typically 3 of these 33
        ax = np.abs(x)
        room = room + 33 * 2.0 ** -11 * (spread(ax @ case.top[0][e]) if case.rot is not None else ax @ case.top[0][e])
        room = room + 33 * 2.0 ** -11 * spread(ax @ case.top[1][e])
        norm += 3 * 2.0 ** -11
    if not back and case.k > 2 ** 15:
        # The quadratic sum above is of K up to 2^15.  An accumulator takes an eighth of the 2 K entries, 32 at a time, in
        # three products: L = 6 K / 256 additions, each off by 2^-24 / sqrt(3) of a partial sum which grows as the root of
        # its terms, sum_i i / L = L / 2: 2^-24 sqrt(L / 6) = 2^-24 sqrt(K / 256) of a typical result.  Four times that: the
        # norm is of a few results only, which may be smaller than typical.
        norm += 4 * 2.0 ** -24 * math.sqrt(case.k / 256)
    d = np.abs(_f64(got) - want)
    assert (d <= HALF_STEP[out] * np.abs(want) + room + LEAST[out]).all(), \
        (d / (HALF_STEP[out] * np.abs(want) + room + LEAST[out])).max()
    rel = np.linalg.norm(d) / max(np.linalg.norm(want), 1e-300)
    assert rel <= norm + HALF_STEP[out], rel


def _product(case, t, dtype, out, back, x_group=0, ldx=None, ldy=None, shift=0, seed=0):
    rng = np.random.default_rng([t, seed])
    wx, wy = (case.m, case.k) if back else (case.k, case.m)
    scales = None
    x = _rows(rng, t, wx, dtype, ldx, shift)
    x64 = _f64(x)
    if dtype == "e4m3":
        cols = -(-wx // x_group) if x_group else 1
        scales = torch.from_numpy(rng.uniform(0.01, 2.0, (t, cols)).astype(np.float32)).cuda()
        x64 = x64 * np.repeat(_f64(scales), x_group or wx, axis=1)[:, :wx]
    flat, y = _buffer(t, wy, out, ldy, shift)
    (K.kashin_matmul_t if back else K.kashin_matmul)(case.plan, *case.dev, x, y, case.work(t, back), scales, x_group,
                                                    rot_seed=case.rot)
    torch.cuda.synchronize()
    f, wide = flat.to(torch.float32), ldy or wy
    assert (f[:shift] == 7).all() and (f[shift + t * wide:] == 7).all()
    assert (f[shift:shift + t * wide].view(t, wide)[:, wy:] == 7).all()
    return x64, y


LENGTHS = [n for n in (64, 96, 172, 256, 512, 768, 1024, 2048, 4096, 5120, 6144, 8192, 10000, 11008, 13824, 14336, 16384)]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("n", LENGTHS)
def test_products_of_every_length(n, back):
    print(f"product n={n} back={back}", flush=True)
    case = Case(n, 37)
    for t, dtype, out in ((1, "f32", "f32"), (3, "bf16", "f32"), (18, "f16", "bf16")):
        x, y = _product(case, t, dtype, out, back)
        _check(case, y, x, out, back)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("t", [1, 2, 4, 5, 8, 15, 16, 17, 31, 33, 64, 65, 130, 257])
@pytest.mark.parametrize("m", [1, 15, 130, 1000])
def test_products_of_row_counts(t, m, back):
    print(f"product t={t} m={m} back={back}", flush=True)
    case = Case(512, m, groups=2)
    for dtype, out in (("bf16", "bf16"), ("f32", "f32"), ("f16", "f16")):
        x, y = _product(case, t, dtype, out, back)
        _check(case, y, x, out, back)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("n,groups,m,rot", [(64, 5, 70, None), (64, 16, 33, 3), (96, 7, 40, 5), (172, 3, 40, 9), (172, 6, 65, None),
                                            (256, 16, 50, None), (1024, 3, 129, 4), (11008, 1, 20, 8), (5120, 2, 30, None),
                                            (10000, 2, 17, None)])
def test_products_of_groups_and_rotations(n, groups, m, rot, back):
    print(f"product n={n} groups={groups} rot={rot} back={back}", flush=True)
    case = Case(n, m, groups, rot=rot)
    for t, dtype, out, xg in ((1, "e4m3", "f32", 0), (6, "e4m3", "f16", 32), (40, "e4m3", "f32", 128), (19, "f32", "f32", 0)):
        x, y = _product(case, t, dtype, out, back, xg)
        _check(case, y, x, out, back)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("n,groups,m,t", [(256, 2, 4100, 1050), (64, 1, 33000, 200), (96, 3, 8200, 511), (512, 1, 2100, 2049), (256, 2, 11000, 195),
                                          (172, 1, 9000, 250)])
def test_products_of_many_rows(n, groups, m, t, back):
    print(f"product n={n} groups={groups} m={m} t={t} back={back}", flush=True)
    case = Case(n, m, groups)
    for dtype, out in (("bf16", "bf16"), ("f32", "f32")):
        x, y = _product(case, t, dtype, out, back)
        _check(case, y, x, out, back)


@pytest.mark.parametrize("n,groups,m,t", [(64, 4096, 3, 1), (64, 4096, 3, 5), (64, 64, 5, 1601), (96, 48, 20, 700)])
def test_products_of_rows_of_many_groups(n, groups, m, t):
    print(f"product n={n} groups={groups} m={m} t={t}", flush=True)
    case = Case(n, m, groups)
    for dtype, out, xg in (("bf16", "bf16", 0), ("e4m3", "f32", 96), ("f32", "f16", 0)):
        x, y = _product(case, t, dtype, out, False, xg, None if t > 5 else case.k + 3)
        _check(case, y, x, out, False)


@pytest.mark.parametrize("n,groups", [(172, 5), (512, 3), (4096, 1)])
@pytest.mark.parametrize("x_group", [32, 96, 160, 4096])
def test_products_of_scales_across_groups(n, groups, x_group):
    """Scales of x whose entries begin and end inside a group of the codes, in both directions."""
    for back in (False, True):
        case = Case(n, 300, groups)
        for t in (1, 2, 70):
            x, y = _product(case, t, "e4m3", "f32", back, x_group)
            _check(case, y, x, "f32", back)


def test_rows_that_are_not_finite_keep_to_themselves():
    """A row of several groups, or of e4m3 scales, next to rows that share its workgroups: they stay right."""
    for n, groups in ((256, 3), (172, 1), (64, 5)):
        case = Case(n, 30, groups)
        x = _rows(np.random.default_rng(n), 9, case.k, "f16")
        q, scales = x.to(torch.float8_e4m3fn), torch.ones((9, 1), device="cuda")
        y = torch.empty((9, 30), device="cuda")
        x[4, case.k - 1] = math.inf
        K.kashin_matmul(case.plan, *case.dev, x, y, case.work(9, False))
        others = [i for i in range(9) if i != 4]
        _check(case, y[others], _f64(x[others]), "f32", False)
        assert y[4].isnan().all()
        scales[2] = math.nan
        K.kashin_matmul(case.plan, *case.dev, q, y, case.work(9, False), scales)
        others = [i for i in range(9) if i != 2]
        _check(case, y[others], _f64(q[others]), "f32", False)
        assert y[2].isnan().all()


@pytest.mark.parametrize("back", [False, True])
def test_experts_of_many_rows(back):
    for out in ("f32", "f16"):
        _experts(Case(256, 4100, 1, experts=5), [150, 0, 900, 128, 33], 1215, "bf16", out, back, 1)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("dtype,out", [("f32", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("e4m3", "bf16")])
def test_products_of_strided_and_unaligned_rows(dtype, out, back):
    case = Case(256, 61, 3)
    for t in (1, 7, 40):
        wx, wy = (case.m, case.k) if back else (case.k, case.m)
        for shift, px, py in ((1, 1, 5), (3, 8, 0), (8, 3, 16)):
            x, y = _product(case, t, dtype, out, back, 64 if dtype == "e4m3" else 0, wx + px, wy + py, shift)
            _check(case, y, x, out, back)


@pytest.mark.parametrize("back", [False, True])
def test_product_magnitudes_over_the_whole_range(back):
    """Rows of x and centres scaled by powers of two give results scaled alike, bit for bit, far from one and close to
    the ends of fp32, also where the factors differ from row to row."""
    case = Case(512, 50)
    x = _rows(np.random.default_rng(1), 20, case.m if back else case.k, "f32")
    y = torch.empty((20, case.k if back else case.m), device="cuda")
    f = K.kashin_matmul_t if back else K.kashin_matmul
    f(case.plan, *case.dev, x, y, case.work(20, back))
    cu, cv, ce = case.dev
    for a, b in ((60, 0), (-60, 10), (0, -70), (100, -100), (-20, 90)):
        z = torch.empty_like(y)
        f(case.plan, cu, cv, ce * 2.0 ** b, x * 2.0 ** a, z, case.work(20, back))
        assert torch.equal(z, y * 2.0 ** (a + b)), (a, b)
    scale = torch.tensor([[2.0 ** e] for e in range(-40, 40, 4)], device="cuda")
    z = torch.empty_like(y)
    f(case.plan, *case.dev, x * scale, z, case.work(20, back))
    assert torch.equal(z, y * scale)


def test_products_of_rows_that_are_not_finite():
    case = Case(256, 40, 2)
    for back in (False, True):
        for t in (3, 50):
            x = _rows(np.random.default_rng(t), t, case.m if back else case.k, "f32")
            x[1, 5], x[2, 7] = math.nan, math.inf
            clean = x.clone()
            clean[1:3] = 0.0
            y, z = (torch.empty((t, case.k if back else case.m), device="cuda") for _ in range(2))
            f = K.kashin_matmul_t if back else K.kashin_matmul
            f(case.plan, *case.dev, x, y, case.work(t, back))
            f(case.plan, *case.dev, clean, z, case.work(t, back))
            torch.cuda.synchronize()
            assert y[1:3].isnan().all()
            keep = [i for i in range(t) if i not in (1, 2)]
            _check(case, y[keep], _f64(clean[keep]), "f32", back)
            assert (z[1:3] == 0).all()


def test_products_of_centres_that_are_not_finite():
    """A row of W_hat (as the quantiser leaves a row that was not finite) gives a column of NaN; in the transposed
    product it reaches the columns of its group."""
    case = Case(256, 40, 2)
    cu, cv, ce = case.dev
    ce = ce.clone()
    ce[7 * 2 + 1] = math.nan
    x = _rows(np.random.default_rng(0), 30, case.k, "f32")
    y = torch.empty((30, 40), device="cuda")
    K.kashin_matmul(case.plan, cu, cv, ce, x, y, case.work(30, False))
    assert y[:, 7].isnan().all()
    keep = [i for i in range(40) if i != 7]
    assert y[:, keep].isfinite().all()
    x = _rows(np.random.default_rng(0), 30, 40, "f32")
    y = torch.empty((30, 512), device="cuda")
    K.kashin_matmul_t(case.plan, cu, cv, ce, x, y, case.work(30, True))
    assert y[:, 256:].isnan().all() and y[:, :256].isfinite().all()


@pytest.mark.parametrize("n,groups,m,rot", [(512, 1, 200, None), (256, 4, 77, 6), (96, 2, 130, None)])
def test_transposed_product_is_the_gradient(n, groups, m, rot):
    """The product is linear in x: its gradient for a given dy is dy W (the formula, checked above) and equals the
    difference <dy, f(x + d) - f(x)> = <dy W, d> along any d, both taken from the kernels' outputs."""
    case = Case(n, m, groups, rot=rot)
    rng = np.random.default_rng(5)
    for t in (1, 9, 80):
        x, d = _rows(rng, t, case.k, "f32"), _rows(rng, t, case.k, "f32")
        dy = _rows(rng, t, m, "f32")
        y0, y1, g = torch.empty((t, m), device="cuda"), torch.empty((t, m), device="cuda"), torch.empty((t, case.k), device="cuda")
        K.kashin_matmul(case.plan, *case.dev, x, y0, case.work(t, False), rot_seed=rot)
        K.kashin_matmul(case.plan, *case.dev, x + d, y1, case.work(t, False), rot_seed=rot)
        K.kashin_matmul_t(case.plan, *case.dev, dy, g, case.work(t, True), rot_seed=rot)
        lhs = (_f64(dy) * (_f64(y1) - _f64(y0))).sum()
        rhs = (_f64(g) * _f64(d)).sum()
        # each result is within NORM of its norm; the difference of two of them twice
        room = NORM * (np.linalg.norm(_f64(dy)) * (np.linalg.norm(_f64(y0)) + np.linalg.norm(_f64(y1))) +
                       np.linalg.norm(_f64(g)) * np.linalg.norm(_f64(d)))
        # and x + d was rounded to fp32
        room += 2.0 ** -24 * np.linalg.norm(_f64(x + d)) * np.linalg.norm(_f64(g))
        assert abs(lhs - rhs) <= room, (lhs, rhs, room)


# ----------------------------------------------------------------------------- experts
def _experts(case, counts, t, dtype, out, back, first=0, seed=0):
    rng = np.random.default_rng([seed, t])
    wx, wy = (case.m, case.k) if back else (case.k, case.m)
    x = _rows(rng, t, wx, dtype)
    scales = None
    x64 = _f64(x)
    if dtype == "e4m3":
        scales = torch.from_numpy(rng.uniform(0.1, 2.0, (t, 1)).astype(np.float32)).cuda()
        x64 = x64 * _f64(scales)
    off = first + np.concatenate([[0], np.cumsum(counts)])
    flat, y = _buffer(t, wy, out)
    K.kashin_matmul_experts(case.plan, *case.dev, torch.from_numpy(off.astype(np.int64)).cuda(), x, y, case.work(t, back), back,
                            scales, 0, rot_seed=case.rot)
    torch.cuda.synchronize()
    for e in range(case.experts):
        _check(case, y[off[e]:off[e + 1]], x64[off[e]:off[e + 1]], "f32" if out == "f32" else out, back, e)
    f = flat.to(torch.float32)
    assert (f[:off[0] * wy] == 7).all() and (f[off[-1] * wy:] == 7).all()  # rows that no expert has


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("counts,spare,first", [([5], 0, 0), ([0, 1, 0, 40, 3], 0, 0), ([16, 16, 32], 2, 0), ([0, 0, 0], 4, 0),
                                                ([1] * 70, 1, 3), ([0] * 64 + [33] + [0] * 64 + [2, 17], 0, 0),
                                                ([200, 3], 5, 2)])
def test_experts(counts, spare, first, back):
    print(f"experts {len(counts)} spare {spare} back={back}", flush=True)
    case = Case(256, 35, 2, experts=len(counts))
    t = first + sum(counts) + spare
    for dtype, out in (("f32", "f32"), ("bf16", "f16"), ("e4m3", "f32")):
        _experts(case, counts, t, dtype, out, back, first)


def test_experts_rotated_and_wide():
    for back in (False, True):
        _experts(Case(1024, 300, 1, experts=4, rot=2), [7, 0, 150, 20], 177, "bf16", "f32", back)


@pytest.mark.parametrize("back", [False, True])
def test_experts_equal_single_products(back):
    """Every expert's rows as kashin_matmul gives them on that expert's matrix alone (to rounding: pairs of rows share a
    transform); offsets beyond the rows are taken as the last row."""
    case = Case(512, 48, experts=3)
    t = 21
    x = _rows(np.random.default_rng(2), t, case.m if back else case.k, "f32")
    y = torch.zeros((t, case.k if back else case.m), device="cuda")
    off = torch.tensor([-4, 6, 6, 1 << 40], device="cuda")
    K.kashin_matmul_experts(case.plan, *case.dev, off, x, y, case.work(t, back), back)
    for e, (lo, hi) in enumerate(((0, 6), (6, 6), (6, t))):
        _check(case, y[lo:hi], _f64(x[lo:hi]), "f32", back, e)


# ----------------------------------------------------------------------------- runs of them together
def test_layer_run():
    """A decoding step's layer as a program runs it: weights quantised by the library, the norm in 8 bits with scales, the
    product from the codes, and the gradient back through it; against W_hat of kashin_reconstruct."""
    torch.manual_seed(0)
    n, m, t = 1024, 768, 12
    plan = K.kashin_plan(n, 5, 12)
    w = torch.randn(m, n, device="cuda") * 0.02
    codes = K.quantize_alloc(plan, w, 1)
    w_hat = torch.empty(m, n, device="cuda")
    K.kashin_reconstruct(plan, *codes, w_hat)
    x, r = torch.randn(t, n, device="cuda").bfloat16(), torch.randn(t, n, device="cuda").bfloat16()
    g = (1 + 0.1 * torch.randn(n, device="cuda")).bfloat16()
    h, q, s = torch.empty_like(x), torch.empty(t, n, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(t, n // 128, device="cuda")
    K.kashin_rmsnorm(x, r, g, 1e-5, h, q, s, 128)
    y = K.matmul_alloc(plan, *codes, q, out_dtype=torch.float32, x_scales=s, x_group=128)
    back = K.matmul_alloc(plan, *codes, y, transposed=True)
    torch.cuda.synchronize()
    xq = _f64(q) * np.repeat(_f64(s), 128, axis=1)
    want = xq @ _f64(w_hat).T
    assert np.linalg.norm(_f64(y) - want) <= 2 * NORM * np.linalg.norm(want)  # and w_hat's own rounding
    want = _f64(y) @ _f64(w_hat)
    assert np.linalg.norm(_f64(back) - want) <= 2 * NORM * np.linalg.norm(want)


def test_codes_held_transposed():
    """Codes that the error-compensated quantisation leaves (rows are W's columns): x W^T of the compensated matrix is the
    transposed product with them."""
    d_in, d_out = 96, 256
    plan = K.kashin_plan(d_out, 3, 8)
    rng = np.random.default_rng(0)
    w_t = torch.from_numpy((rng.standard_normal((d_in, d_out)) * 0.02).astype(np.float32)).cuda()
    h = torch.from_numpy(ref.synthetic_hessian(d_in, 300, 1).astype(np.float32)).cuda()
    cu, cv, ce, q_t = optq.optq_quantize(plan, w_t, h, chunk=32)
    x = _rows(rng, 7, d_in, "f32")
    y = K.matmul_alloc(plan, cu, cv, ce, x, transposed=True)
    want = _f64(x) @ _f64(q_t)
    assert np.linalg.norm(_f64(y) - want) <= 2 * NORM * np.linalg.norm(want)


def test_captured_layer_replays():
    """Norm, product, transposed and grouped products in one captured graph, two graphs with workspaces of their own:
    every replay as the eager calls, bit for bit, with eager work and other inputs in between."""
    case, ex = Case(512, 300, 2), Case(256, 64, 2, experts=5)
    t = 20
    rng = np.random.default_rng(0)
    off = torch.tensor([0, 3, 3, 10, 19, 20], device="cuda")

    def state():
        return {"x": _rows(rng, t, 1024, "bf16"), "h": torch.empty((t, 1024), dtype=torch.bfloat16, device="cuda"),
                "q": torch.empty((t, 1024), dtype=torch.float8_e4m3fn, device="cuda"),
                "s": torch.empty((t, 8), device="cuda"), "y": torch.empty((t, 300), device="cuda"),
                "z": torch.empty((t, 1024), device="cuda"), "e": torch.zeros((t, 64), device="cuda"),
                "et": torch.zeros((t, 512), device="cuda"),
                "work": [case.work(t, False), case.work(t, True), ex.work(t, False), ex.work(t, True)]}

    def step(s):
        K.kashin_rmsnorm(s["x"], s["h"], None, 1e-5, s["h"], s["q"], s["s"], 128)
        K.kashin_matmul(case.plan, *case.dev, s["q"], s["y"], s["work"][0], s["s"], 128)
        K.kashin_matmul_t(case.plan, *case.dev, s["y"], s["z"], s["work"][1])
        K.kashin_matmul_experts(ex.plan, *ex.dev, off, s["z"][:, :512], s["e"], s["work"][2])
        K.kashin_matmul_experts(ex.plan, *ex.dev, off, s["e"], s["et"], s["work"][3], True)

    states, graphs = [state(), state()], []
    eager = state()
    for s in states + [eager]:
        s["h"].zero_()
    step(eager)
    torch.cuda.synchronize()
    for s in states:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(s)
        graphs.append(g)
    for i in range(4):
        for s, g in zip(states, graphs):
            x, h = _rows(rng, t, 1024, "bf16"), _rows(rng, t, 1024, "bf16")
            s["x"].copy_(x)
            s["h"].copy_(h)
            eager["x"].copy_(x)
            eager["h"].copy_(h)
            g.replay()
            step(eager)
            torch.cuda.synchronize()
            for key in ("h", "q", "s", "y", "z", "e", "et"):
                assert torch.equal(s[key].view(torch.uint8), eager[key].view(torch.uint8)), (i, key)


def test_products_on_two_streams_repeat():
    """Calls on two streams at once, each with its own workspace: the results of calls alone, bit for bit."""
    case = Case(1024, 500)
    x = [_rows(np.random.default_rng(i), 9 + 30 * i, 1024, "f16") for i in range(2)]
    alone = [K.matmul_alloc(case.plan, *case.dev, v) for v in x]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in x]
    work = [case.work(v.shape[0], False) for v in x]
    ys = [torch.empty_like(a) for a in alone]
    torch.cuda.synchronize()
    for _ in range(5):
        for v, y, w, s in zip(x, ys, work, streams):
            K.kashin_matmul(case.plan, *case.dev, v, y, w, stream=s)
    torch.cuda.synchronize()
    for y, a in zip(ys, alone):
        assert torch.equal(y, a)


def test_product_refusals_with_a_plan():
    case = Case(320 if K.kashin_supported_n(320) else 5120, 4)
    n = case.n
    x, y, work = torch.zeros((2, n), device="cuda"), torch.zeros((2, 4), device="cuda"), case.work(2, False)

    def refused(match, **kw):
        a = {"x": x, "y": y, "work": work, "rot_seed": None, "x_scales": None, "x_group": 0}
        a.update(kw)
        with pytest.raises((K.KashinError, ValueError, TypeError), match=match):
            K.kashin_matmul(case.plan, *case.dev, **a)

    refused("odd part", rot_seed=3)
    refused("work must hold", work=work[:-16])
    refused("16-byte", work=torch.empty(work.numel() + 8, dtype=torch.uint8, device="cuda")[8:])
    refused("overlap", y=x[:, :4])
    refused("overlap", y=work[: 2 * 4 * 4].view(torch.float32).view(2, 4))
    refused("x_scales", x=x.to(torch.float8_e4m3fn))
    refused("x_scales", x_scales=torch.zeros((2, 1), device="cuda"))
    refused("multiple of 32", x=x.to(torch.float8_e4m3fn), x_group=48, x_scales=torch.zeros((2, -(-n // 48)), device="cuda"))
    refused("dtype", y=y.to(torch.float64))
    refused("dtype", y=y.to(torch.float8_e4m3fn))
    refused("shape", y=torch.zeros((3, 4), device="cuda"))
    refused("columns", x=torch.zeros((2, n - 4), device="cuda"))
    refused("live on", x=torch.zeros((2, n)))
    L = K.lib()
    w = K.Weights(case.plan.handle, None, *(t.data_ptr() for t in case.dev), 4, 1, 2)
    import ctypes
    args = (x.data_ptr(), 0, 2, n, None, 0, y.data_ptr(), 0, 4, work.data_ptr(), work.numel(), None)
    assert L.kashin_matmul(ctypes.addressof(w), *args) == K.KASHIN_E_INVALID  # experts
    w.experts = 1
    w.m = 0
    assert L.kashin_matmul(ctypes.addressof(w), *args) == K.KASHIN_E_INVALID
    w.m, w.groups = 4, (1 << 20) // n + 1
    assert L.kashin_matmul(ctypes.addressof(w), *args) == K.KASHIN_E_INVALID
    w.groups = 1
    assert L.kashin_matmul_experts(ctypes.addressof(w), None, 0, *args) == K.KASHIN_E_INVALID  # no offsets
    assert L.kashin_matmul_experts(ctypes.addressof(w), x.data_ptr(), 2, *args) == K.KASHIN_E_INVALID
    short = (x.data_ptr(), 0, 2, n - 1) + args[4:]
    assert L.kashin_matmul(ctypes.addressof(w), *short) == K.KASHIN_E_INVALID
    # no rows: nothing is looked at
    empty = (None, 0, 0, n, None, 0, None, 0, 4, None, 0, None)
    assert L.kashin_matmul(ctypes.addressof(w), *empty) == K.KASHIN_OK
    K.kashin_matmul(case.plan, *case.dev, x[:0], y[:0], work[:0])


def test_outputs_over_other_arguments_are_refused():
    case = Case(512, 6, experts=2)
    cu, cv, ce = case.dev
    x, y = torch.zeros((4, 512), device="cuda"), torch.zeros((4, 6), device="cuda")
    off = torch.tensor([0, 2, 4], device="cuda")
    work = case.work(4, False)
    before = [a.clone() for a in (cu, cv, ce, off)]
    q = x.to(torch.float8_e4m3fn)
    for over in (cu.view(-1)[:96].view(torch.float32).view(4, 6), ce.view(-1)[8:32].view(4, 6)):
        with pytest.raises((K.KashinError, ValueError), match="overlap"):
            K.kashin_matmul_experts(case.plan, cu, cv, ce, off, x, over, work, False)
    big = torch.zeros(work.numel() + 4096, dtype=torch.uint8, device="cuda")
    inside = big[256:272].view(torch.float32).view(4, 1)
    with pytest.raises((K.KashinError, ValueError), match="overlap"):
        K.kashin_matmul_experts(case.plan, cu, cv, ce, off, q, y, big, False, inside)
    o2 = big[512:536].view(torch.int64)
    with pytest.raises((K.KashinError, ValueError), match="overlap"):
        K.kashin_matmul_experts(case.plan, cu, cv, ce, o2, x, y, big, False)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, (cu, cv, ce, off)))
