"""The performance cases of the operators that serve (and train adapters on) a quantised model's layers.

    rmsnorm     the residual's addition and the root-mean-square norm before a layer, with an 8-bit output
                (e4m3 with a scale for each row or group of entries) or one in the model's type
    matmul      Y = X W^T for W held as 2 + 2 bit codes with group centres (W = U + V P, P the plan's operator):
                one token, a batch of decoding sequences, a prompt
    matmul_t    Y = X W: the product for codes held transposed, and the gradient of matmul's input
    experts     both of them grouped by expert, ragged row counts between device offsets

    listed()           the named cases
    draw(rng)          one more case of the same ranges
    prepare(case, s)   inputs, plan and buffers, from the seed alone
    run(state)         one pass: the plain form, or the library's calls where `own` is set
    work(case)         bytes and flops the pass cannot do without
    exact(case, s)     the outputs in float64
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
SIZES = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}
E4M3_MAX = 448.0


def listed():
    return [
        # one decoding sequence at the norm before an attention layer (the smallest call)
        {"name": "norm 1x4096", "op": "rmsnorm", "t": 1, "n": 4096, "dtype": "bf16", "out": "e4m3", "group": 128,
         "residual": 1},
        # a batch of sequences, a width that is no multiple of anything, one scale a row
        {"name": "norm 193x5003", "op": "rmsnorm", "t": 193, "n": 5003, "dtype": "f16", "out": "e4m3", "group": 0,
         "residual": 1},
        # a prompt's rows, the norm's output in the model's type (the largest norm)
        {"name": "norm 8192x8192", "op": "rmsnorm", "t": 8192, "n": 8192, "dtype": "bf16", "out": "bf16", "group": 0,
         "residual": 1},
        # one token through the MLP input matrix of a 7B-sized layer
        {"name": "matmul 1x4096->11008", "op": "matmul", "t": 1, "n": 4096, "groups": 1, "m": 11008, "dtype": "bf16",
         "out": "bf16", "rot": 0},
        # a batch of eleven sequences through the MLP output matrix, rotated weights, rows of a float32 program
        {"name": "matmul 11x11008->4096 +H", "op": "matmul", "t": 11, "n": 11008, "groups": 1, "m": 4096,
         "dtype": "f32", "out": "f32", "rot": 1},
        # one token, 8-bit activations with scales, centres for each 256 weights
        {"name": "matmul 1x4096->4096 g256", "op": "matmul", "t": 1, "n": 256, "groups": 16, "m": 4096,
         "dtype": "e4m3", "out": "f16", "rot": 0},
        # a prompt through the MLP input matrix (the largest product)
        {"name": "matmul 2048x4096->11008", "op": "matmul", "t": 2048, "n": 4096, "groups": 1, "m": 11008,
         "dtype": "bf16", "out": "bf16", "rot": 0},
        # one token through a matrix whose codes are held transposed (error-compensated quantisation)
        {"name": "matmul_t 1x4096->4096", "op": "matmul_t", "t": 1, "n": 4096, "groups": 1, "m": 4096,
         "dtype": "f16", "out": "f16", "rot": 0},
        # the gradient of a batch of training rows with respect to the MLP input
        {"name": "matmul_t 509x11008->4096", "op": "matmul_t", "t": 509, "n": 4096, "groups": 1, "m": 11008,
         "dtype": "bf16", "out": "bf16", "rot": 0},
        # sixteen sequences decoding through two of eight experts each
        {"name": "experts 8: 32x4096->2048", "op": "experts", "experts": 8, "t": 32, "tail": 0, "n": 4096,
         "groups": 1, "m": 2048, "dtype": "e4m3", "out": "bf16", "rot": 0, "transposed": 0},
        # a prompt's rows over many small experts, some without rows, spare rows behind the last
        {"name": "experts 64: 4000x2048->1000", "op": "experts", "experts": 64, "t": 4000, "tail": 77, "n": 2048,
         "groups": 1, "m": 1000, "dtype": "bf16", "out": "bf16", "rot": 0, "transposed": 0},
        # the gradient of the experts' rows
        {"name": "experts 8 t: 700x2048->4096", "op": "experts", "experts": 8, "t": 700, "tail": 0, "n": 4096,
         "groups": 1, "m": 2048, "dtype": "bf16", "out": "f32", "rot": 0, "transposed": 1},
    ]


WIDTHS = (64, 96, 172, 256, 512, 768, 1024, 2048, 4096, 5120, 6144, 8192, 10000, 11008, 13824, 14336, 16384)
MOST_PRODUCTS = 2048 * 4096 * 11008


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rmsnorm", "matmul", "matmul", "matmul_t", "experts"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op == "rmsnorm":
        n = _log_int(rng, 64, 16384)
        if rng.randrange(3):
            n = -(-n // 64) * 64
        out = rng.choice(["e4m3", "e4m3", dtype])
        return {"op": op, "t": _log_int(rng, 1, 8192 * 8192 // n if n > 8192 else 8192), "n": n, "dtype": dtype,
                "out": out, "group": rng.choice([0, 32, 64, 128, 256]) if out == "e4m3" else 0,
                "residual": int(rng.randrange(4) > 0)}
    n = rng.choice(WIDTHS)
    groups = rng.randint(1, max(1, min(16, 4096 // n)))
    rot = int(n // (n & -n) in (1, 3, 43) and rng.randrange(4) == 0)
    m = _log_int(rng, 64, 16384)
    out = rng.choice(["f32", "f16", "bf16"])
    c = {"op": op, "n": n, "groups": groups, "m": m, "dtype": rng.choice([dtype, dtype, "e4m3"]), "out": out, "rot": rot}
    k = n * groups
    if op == "experts":
        c["experts"] = _log_int(rng, 2, max(2, min(64, 1.5e8 / (m * k))))
        c["t"] = _log_int(rng, 1, min(4096, MOST_PRODUCTS / (m * k)))
        c["tail"] = rng.choice([0, 0, 5])
        c["transposed"] = rng.randrange(2)
    else:
        c["t"] = _log_int(rng, 1, min(2048, MOST_PRODUCTS / (m * k)))
    return c


# ----------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _activations(g, m, n):
    """m x n fp32 activations, N(0, 1) with 0.1 % of the channels scaled by 20."""
    x = torch.randn((m, n), generator=g, device="cuda")
    x[:, torch.randperm(n, generator=g, device="cuda")[: max(1, n // 1000)]] *= 20.0
    return x


def _codes(g, m, n):
    """Packed 2-bit codes and centres of m rows of n: inner centres twice as frequent as outer ones, centres +-c1 +- c2
    as two greedy steps on weights of standard deviation 0.02 leave them, moved a little as k-means does."""
    p = torch.randint(0, 6, (2, m, n // 4, 4), generator=g, device="cuda", dtype=torch.uint8)
    c = (p > 0).to(torch.uint8) + (p > 2) + (p > 4)
    packed = c[..., 0] | (c[..., 1] << 2) | (c[..., 2] << 4) | (c[..., 3] << 6)
    s = 0.8 + 0.4 * torch.rand((m, 2, 4), generator=g, device="cuda")
    q = torch.tensor([[-0.023, -0.005, 0.005, 0.023], [-0.007, -0.002, 0.002, 0.007]], device="cuda")
    return packed[0].contiguous(), packed[1].contiguous(), (q * s).contiguous()


def _counts(seed, experts, rows):
    """Ragged row counts of the experts: shares spread over a factor of about fifty, some of them zero."""
    r = np.random.default_rng(int(seed))
    share = np.exp(r.normal(0.0, 1.0, experts)) * (r.random(experts) > 0.1)
    if not share.any():
        share[0] = 1.0
    return r.multinomial(rows, share / share.sum())


def _signs(count, seed):
    """+-1 from the top bits of splitmix64's outputs from `seed`."""
    i = np.arange(1, count + 1, dtype=np.uint64)
    with np.errstate(over="ignore"):
        z = np.uint64(seed) + i * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z ^= z >> np.uint64(31)
    return torch.from_numpy(np.where(z >> np.uint64(63), -1.0, 1.0)).to("cuda")


def _dct(n):
    """The orthonormal DCT-II matrix in 64 bits, rows k, columns i, angles reduced in integers."""
    k = torch.arange(n, device="cuda")[:, None]
    a = ((2 * torch.arange(n, device="cuda") + 1)[None, :] * k) % (4 * n)
    c = torch.cos(a.to(torch.float64) * (math.pi / (2 * n))) * math.sqrt(2.0 / n)
    c[0] *= math.sqrt(0.5)
    return c


def _hadamard(size):
    i = torch.arange(size, device="cuda")
    x = i[:, None] & i[None, :]
    x = x ^ (x >> 8)
    x = x ^ (x >> 4)
    x = x ^ (x >> 2)
    x = x ^ (x >> 1)
    return 1.0 - 2.0 * (x & 1).to(torch.float64)


def _seeds(seed):
    """The plan's sign seed and the rotation's."""
    return int(seed) % (1 << 40) + 1, int(seed) % (1 << 40) + 5


def _x_of(case, g, t, width):
    """The rows and, for 8-bit ones, their scales for each 128 entries."""
    x = _activations(g, t, width)
    if case["dtype"] != "e4m3":
        return x.to(DTYPES[case["dtype"]]), None
    groups = -(-width // 128)
    pad = torch.zeros((t, groups * 128), device="cuda")
    pad[:, :width] = x
    scales = pad.reshape(t, groups, 128).abs().amax(-1) / E4M3_MAX
    q = pad.reshape(t, groups, 128) / scales[..., None]
    return q.reshape(t, -1)[:, :width].clamp(-E4M3_MAX, E4M3_MAX).to(DTYPES["e4m3"]).contiguous(), scales


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    st = {"case": dict(case)}
    if op == "rmsnorm":
        t, n, dt = case["t"], case["n"], DTYPES[case["dtype"]]
        st["x"] = _activations(g, t, n).to(dt)
        st["r"] = (2.0 * _activations(g, t, n)).to(dt) if case["residual"] else None
        st["w"] = (1.0 + 0.2 * torch.randn(n, generator=g, device="cuda")).to(dt)
        st["h"] = torch.empty((t, n), dtype=dt, device="cuda") if case["residual"] else None
        st["y"] = torch.empty((t, n), dtype=DTYPES[case["out"]], device="cuda")
        st["s"] = torch.empty((t, -(-n // case["group"]) if case["group"] else 1), device="cuda") \
            if case["out"] == "e4m3" else None
        if own:
            from paper_2609_11687_amd import kashin

            st["lib"] = kashin
        return st
    n, groups, m, t = case["n"], case["groups"], case["m"], case["t"] + case.get("tail", 0)
    experts, back = case.get("experts", 1), op == "matmul_t" or case.get("transposed", 0)
    k = n * groups
    st["codes"] = _codes(g, experts * m * groups, n)
    st["x"], st["xs"] = _x_of(case, g, t, m if back else k)
    st["y"] = torch.zeros((t, k if back else m), dtype=DTYPES[case["out"]], device="cuda")
    counts = _counts(seed, experts, case["t"])
    st["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)).to("cuda")
    st["most"] = int(counts.max())
    sign_seed, rot_seed = _seeds(seed)
    st["rot"] = rot_seed if case["rot"] else None
    if own:
        from paper_2609_11687_amd import kashin

        st["lib"] = kashin
        st["plan"] = kashin.kashin_plan(n, sign_seed, 1)
        st["work"] = torch.empty(kashin.kashin_matmul_workspace_bytes(n, m, groups, t, experts, back), dtype=torch.uint8,
                                 device="cuda")
    else:
        c = _dct(n)
        st["P"] = (c.t().contiguous() @ (c * _signs(n, sign_seed)[:, None])).to(torch.float32)
        if case["rot"]:
            b = n // (n & -n)
            r = torch.kron(_hadamard(n // b) / math.sqrt(n // b), _dct(b)) * _signs(n, rot_seed)
            st["R"] = r.to(torch.float32).contiguous()
    return st


# ----------------------------------------------------------------------------- one pass
def run(st):
    if own:
        return _library(st)
    if st["case"]["op"] == "rmsnorm":
        return _plain_norm(st)
    return _plain_product(st)


def _library(st):
    case, lib = st["case"], st["lib"]
    if case["op"] == "rmsnorm":
        lib.kashin_rmsnorm(st["x"], st["r"], st["w"], 1e-5, st["h"], st["y"], st["s"], group=case["group"])
        return {"h": st["h"], "y": st["y"], "s": st["s"]}
    more = {"x_scales": st["xs"], "x_group": 128 if st["xs"] is not None else 0, "rot_seed": st["rot"]}
    if case["op"] == "experts":
        lib.kashin_matmul_experts(st["plan"], *st["codes"], st["offsets"], st["x"], st["y"], st["work"],
                                  transposed=bool(case["transposed"]), **more)
    elif case["op"] == "matmul":
        lib.kashin_matmul(st["plan"], *st["codes"], st["x"], st["y"], st["work"], **more)
    else:
        lib.kashin_matmul_t(st["plan"], *st["codes"], st["x"], st["y"], st["work"], **more)
    return st["y"]


def _plain_norm(st):
    case = st["case"]
    v = st["x"].to(torch.float32)
    h = None
    if st["r"] is not None:
        v = v + st["r"].to(torch.float32)
        h = v.to(st["x"].dtype)
    y = v * torch.rsqrt((v * v).mean(1, keepdim=True) + 1e-5) * st["w"].to(torch.float32)
    if case["out"] != "e4m3":
        return {"h": h, "y": y.to(DTYPES[case["out"]]), "s": None}
    t, n = y.shape
    size = case["group"] or n
    groups = -(-n // size)
    y = torch.cat([y, y.new_zeros((t, groups * size - n))], 1).reshape(t, groups, size)
    s = y.abs().amax(2) / E4M3_MAX
    q = torch.where(s[..., None] > 0, y / s[..., None], 0.0).clamp(-E4M3_MAX, E4M3_MAX)
    return {"h": h, "y": q.reshape(t, -1)[:, :n].to(DTYPES["e4m3"]).contiguous(), "s": s}


def _values(codes, centers):
    """The factor's values in 32 bits: rows x n."""
    c = torch.stack([codes & 3, (codes >> 2) & 3, (codes >> 4) & 3, codes >> 6], 2).reshape(codes.shape[0], -1)
    return centers.gather(1, c.to(torch.int64))


def _widened(x, scales):
    if scales is None:
        return x.to(torch.float32)
    return x.to(torch.float32) * scales.repeat_interleave(128, 1)[:, : x.shape[1]]


def _plain_product(st):
    case = st["case"]
    n, groups, m, experts = case["n"], case["groups"], case["m"], case.get("experts", 1)
    cu, cv, ce = st["codes"]
    u = _values(cu, ce[:, 0]).reshape(experts, m, groups * n)
    v = _values(cv, ce[:, 1]).reshape(experts, m, groups * n)
    x = _widened(st["x"], st["xs"])
    t = x.shape[0]
    back = case["op"] == "matmul_t" or case.get("transposed", 0)

    def spread(a):  # the rows of each expert side by side: experts x most x width
        if case["op"] != "experts":
            return a[None]
        b = a.new_zeros((experts, st["most"], a.shape[1]))
        b[of, at] = a[: case["t"]]
        return b

    def gathered(b):
        return b[of, at] if case["op"] == "experts" else b[0]

    rows = torch.arange(case["t"], device="cuda")
    of = torch.searchsorted(st["offsets"], rows, right=True) - 1
    at = rows - st["offsets"][of]
    if back:
        b = spread(x)
        zu, zv = gathered(b @ u), gathered(b @ v)
        z = zu + (zv.reshape(-1, n) @ st["P"]).reshape(zv.shape)
        y = (z.reshape(-1, n) @ st["R"]).reshape(z.shape) if case["rot"] else z
    else:
        xr = (x.reshape(-1, n) @ st["R"].t()).reshape(x.shape) if case["rot"] else x
        xp = (xr.reshape(-1, n) @ st["P"]).reshape(x.shape)
        y = gathered(spread(xr) @ u.transpose(1, 2) + spread(xp) @ v.transpose(1, 2))
    y = y.to(DTYPES[case["out"]])
    return y if t == case["t"] else torch.cat([y, st["y"][case["t"]:]])


# ----------------------------------------------------------------------------- work
def work(case):
    """Inputs read once, outputs written once.  A product's flops: 2 for each pair of row and weight (W whole) and
    2.5 n log2 n for each of the transforms of P on the rows' groups; the rotation's additions are left out."""
    t, n, size = case["t"], case["n"], SIZES[case["dtype"]]
    if case["op"] == "rmsnorm":
        nbytes = t * n * (size * (3 if case["residual"] else 1) + SIZES[case["out"]]) + n * size
        if case["out"] == "e4m3":
            nbytes += 4 * t * (-(-n // case["group"]) if case["group"] else 1)
        return {"bytes": float(nbytes), "flops": 6.0 * t * n}
    m, groups, experts = case["m"], case["groups"], case.get("experts", 1)
    k = n * groups
    back = case["op"] == "matmul_t" or case.get("transposed", 0)
    wx, wy = (m, k) if back else (k, m)
    # an expert without rows need not be read: at most one expert a row
    nbytes = min(experts, t) * m * groups * (n / 2 + 32) + t * (wx * size + wy * SIZES[case["out"]])
    if case["dtype"] == "e4m3":
        nbytes += 4 * t * -(-wx // 128)
    return {"bytes": float(nbytes), "flops": 2.0 * t * m * k + t * groups * 2 * 2.5 * n * math.log2(n)}


# ----------------------------------------------------------------------------- float64
def _transform64(x, seed):
    """Rows of x (.., n) through DCT-II, the signs and the inverse transform, by a complex FFT of the rows' even and odd
    entries in 64 bits."""
    n = x.shape[-1]
    order = torch.cat([torch.arange(0, n, 2, device="cuda"), torch.arange(n - 1, 0, -2, device="cuda")])
    k = torch.arange(n, device="cuda", dtype=torch.float64)
    turn = torch.polar(torch.ones_like(k), -math.pi * k / (2 * n))
    norm = torch.full((n,), math.sqrt(2.0 / n), dtype=torch.float64, device="cuda")
    norm[0] = math.sqrt(1.0 / n)
    c = (torch.fft.fft(x[..., order]) * turn).real * norm
    c = c * _signs(n, seed) / norm
    flipped = torch.cat([torch.zeros_like(c[..., :1]), c[..., 1:].flip(-1)], -1)
    z = torch.fft.ifft((c - 1j * flipped) * turn.conj()).real
    y = torch.empty_like(z)
    y[..., order] = z
    return y


def _rotate64(x, seed, inverse):
    """R x or R^T x of the rows, R = (Hadamard / sqrt(2^a) kron DCT-II of the odd part) diag(signs)."""
    n = x.shape[-1]
    b = n // (n & -n)
    s, c = _signs(n, seed), _dct(b)
    y = (x if inverse else x * s).reshape(-1, n // b, b)
    y = y @ (c if inverse else c.t()).contiguous()
    h = 1
    while h < n // b:
        y = y.reshape(-1, n // (2 * h * b), 2, h * b)
        y = torch.stack([y[:, :, 0] + y[:, :, 1], y[:, :, 0] - y[:, :, 1]], 2)
        h *= 2
    y = y.reshape(x.shape) / math.sqrt(n // b)
    return y * s if inverse else y


def exact(case, seed):
    """What run() returns, in float64: the weights are put together whole (u + P v, rotated back) and multiplied; an
    8-bit output's values are those before their rounding."""
    st, f = prepare(case, seed), torch.float64
    if case["op"] == "rmsnorm":
        v = st["x"].to(f) + (st["r"].to(f) if st["r"] is not None else 0.0)
        h = v if st["r"] is not None else None
        y = v / torch.sqrt(v.square().mean(1, keepdim=True) + 1e-5) * st["w"].to(f)
        if case["out"] != "e4m3":
            return {"h": h, "y": y, "s": None}
        size = case["group"] or case["n"]
        parts = [p for p in y.split(size, 1)]
        s = torch.stack([p.abs().amax(1) for p in parts], 1) / E4M3_MAX
        return {"h": h, "y": torch.cat([p / s[:, i:i + 1] for i, p in enumerate(parts)], 1), "s": s}
    n, groups, m, experts = case["n"], case["groups"], case["m"], case.get("experts", 1)
    if case["t"] * m * n * groups > 3 * MOST_PRODUCTS:
        return None
    sign_seed, rot_seed = _seeds(seed)
    x = st["x"].to(f)
    if st["xs"] is not None:
        x = torch.cat([p * st["xs"][:, i:i + 1].to(f) for i, p in enumerate(x.split(128, 1))], 1)
    back = case["op"] == "matmul_t" or case.get("transposed", 0)
    out = st["y"].to(f)
    cu, cv, ce = st["codes"]
    bounds = st["offsets"].tolist()
    for e in range(experts):
        if bounds[e] == bounds[e + 1]:
            continue
        rows = slice(e * m * groups, (e + 1) * m * groups)
        parts = []
        for codes, q in ((cu[rows], ce[rows, 0].to(f)), (cv[rows], ce[rows, 1].to(f))):
            w = torch.zeros((m * groups, n), dtype=f, device="cuda")
            for i in range(4):
                c = (codes >> (2 * i)) & 3
                for j in range(4):
                    w[:, i::4] += (c == j) * q[:, j:j + 1]
            parts.append(w)
        w = parts[0] + torch.cat([_transform64(p, sign_seed) for p in parts[1].split(1024)])
        if case["rot"]:
            w = torch.cat([_rotate64(p, rot_seed, True) for p in w.split(1024)])
        w = w.reshape(m, groups * n)
        part = x[bounds[e]:bounds[e + 1]]
        out[bounds[e]:bounds[e + 1]] = part @ w if back else part @ w.t()
    return out
