"""The operators of the 8-bit training and serving path whose speed is followed: the norm before a linear layer and its
backward pass, activations kept in 8 bits, the 8-bit product with a scale for each block of 128, and the weight
gradient taken from an 8-bit checkpoint.

A case is a dict of plain values with a ``kind``:

``norm``      y, statistics = norm(x): layer norm, or RMS norm when ``rms``; ``q8``: y leaves in 8 bits and is returned
              as the values it stands for, in x's type
``norm_bwd``  dx, dgamma (and dbeta) from dy, x and the forward's statistics; ``q8``: x is an 8-bit checkpoint
``ckpt``      an activation saved in 8 bits and restored to its type
``linear``    Y = X W^T for a 16-bit X, which the call turns into 8 bits, and an 8-bit W; with ``dx`` the same for
              the input gradient dX = dY W (W [n, k] in both; M rows)
``grad_w``    dW = dY^T X from an 8-bit checkpoint of X: all of it, or with ``mask`` the two of four consecutive
              positions that a 2:4 pattern keeps

8-bit values are e4m3 (OCP; 3 mantissa bits, largest 448) with one power of two 2^e for each group of 128 consecutive
values of a row (for weights: for each block of 128 x 128), e the smallest integer >= -126 for which the group's largest
magnitude / 2^e does not pass 448. Values past the last column count as zero.
"""
import torch

own = False     # False: the plain form (elementary torch operations in 32 bits); True: the library's entry points

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-5


def listed():
    return [
        # one user's decoding step before a 7B attention projection: the smallest call, all latency
        {"name": "norm_1", "kind": "norm", "m": 1, "k": 4096, "dtype": "bf16", "rms": True, "q8": True, "params": "bf16"},
        # the norm of a 13B block over a ragged batch of prompts, kept in 16 bits
        {"name": "norm_2047", "kind": "norm", "m": 2047, "k": 5120, "dtype": "fp16", "rms": False, "q8": False,
         "params": "fp32"},
        # a training batch on a 70B block: the norm writes the next layer's 8-bit input at once
        {"name": "norm_8192_q8", "kind": "norm", "m": 8192, "k": 8192, "dtype": "bf16", "rms": False, "q8": True,
         "params": "fp32"},
        # a small model's norm backward over a few odd sequences, from an 8-bit checkpoint of its input
        {"name": "norm_bwd_333_q8", "kind": "norm_bwd", "m": 333, "k": 1000, "dtype": "fp16", "rms": False, "q8": True,
         "params": "fp32"},
        # the 70B block's norm backward over a training batch
        {"name": "norm_bwd_8192", "kind": "norm_bwd", "m": 8192, "k": 8192, "dtype": "bf16", "rms": False, "q8": False,
         "params": "fp32"},
        # a short odd activation saved and restored: rows that end inside a group and start off alignment
        {"name": "ckpt_100", "kind": "ckpt", "m": 100, "k": 4097, "dtype": "fp16"},
        # the 70B MLP's widest activation over a training batch
        {"name": "ckpt_8192", "kind": "ckpt", "m": 8192, "k": 28672, "dtype": "bf16"},
        # one user's decoding on a 7B attention projection
        {"name": "linear_1", "kind": "linear", "m": 1, "n": 4096, "k": 4096, "dtype": "bf16", "out": "bf16", "dx": False},
        # a ragged batch of 45 decoding on a 13B gate projection
        {"name": "linear_45", "kind": "linear", "m": 45, "n": 13824, "k": 5120, "dtype": "fp16", "out": "fp16",
         "dx": False},
        # the 70B MLP's input gradient over a training batch: the largest
        {"name": "linear_dx_8192", "kind": "linear", "m": 8192, "n": 28672, "k": 8192, "dtype": "bf16", "out": "bf16",
         "dx": True},
        # a small odd layer's dense weight gradient
        {"name": "grad_w_999", "kind": "grad_w", "m": 999, "n": 2051, "k": 768, "dtype": "fp16", "mask": False},
        # the 70B MLP's weight gradient at its 2:4 mask
        {"name": "grad_w_8192", "kind": "grad_w", "m": 8192, "n": 28672, "k": 8192, "dtype": "bf16", "mask": True},
    ]


def _log(rng, lo, hi):
    return lo * (hi / lo) ** rng.random()


def _size(rng, lo, hi):
    """A width over lo .. hi: any number, or a multiple of 16 or 128 as layers mostly have them."""
    v, mult = int(_log(rng, lo, hi)), rng.choice([1, 16, 128, 128])
    return max(mult, v // mult * mult)


def draw(rng):
    """One more case of the listed ranges, no larger than the largest listed one."""
    kind = rng.choice(["norm", "norm", "norm_bwd", "norm_bwd", "ckpt", "linear", "linear", "linear", "grad_w", "grad_w"])
    k = _size(rng, 128, 28672)
    m = int(_log(rng, 1, 8193))
    if kind in ("norm", "norm_bwd"):
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        return {"kind": kind, "m": min(m, 8192 * 8192 // k), "k": k, "dtype": dtype, "rms": rng.random() < 0.4,
                "q8": dtype != "fp32" and rng.random() < 0.5, "params": rng.choice(["fp32", dtype])}
    if kind == "ckpt":
        return {"kind": kind, "m": min(m, 8192), "k": k, "dtype": rng.choice(["bf16", "fp16", "fp32"])}
    n = _size(rng, 128, 28672)
    m = max(1, min(m, 8192, 8192 * 28672 * 8192 // (n * k)))
    if kind == "linear":
        return {"kind": kind, "m": m, "n": n, "k": k, "dtype": rng.choice(["bf16", "bf16", "fp16"]),
                "out": rng.choice(["bf16", "fp16"]), "dx": rng.random() < 0.4}
    mask = rng.random() < 0.5
    # gradients are taken over whole batches of tokens; a 2:4 pattern is kept in words of 16 positions
    return {"kind": kind, "m": min(max(64, m), 8192 * 28672 * 8192 // (n * k)), "n": n, "k": max(16, k // 16 * 16) if mask else k,
            "dtype": rng.choice(["bf16", "bf16", "fp16"]), "mask": mask}


# --------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _up(a, b):
    return -(-a // b) * b


def _normal(g, shape, std):
    return torch.randn(shape, device="cuda", generator=g) * std


def _act(g, m, k):
    """Activations of order one with one channel in a hundred twenty times larger and an offset of each channel's own."""
    x = _normal(g, (m, k), 1.0)
    x += 0.25 + _normal(g, (k,), 0.3)
    if k >= 100:
        x[:, torch.randperm(k, device="cuda", generator=g)[: k // 100]] *= 20.0
    return x


def _exponents(a):
    """Biased exponent bytes (e + 127) of groups with the largest finite magnitudes `a` (fp32)."""
    return (((a.view(torch.int32) + 0x1FFFFF) >> 23) - 8).clamp(min=1)


def _pow2(b):
    """2^(b - 127) in fp32 from biased exponents 1 .. 254."""
    return (b.to(torch.int32) << 23).view(torch.float32)


def _finite_abs(x):
    return torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))


def _quant(x):
    """Rows of x in 8 bits: codes uint8 [m, k to a multiple of 128], biased exponents uint8 [m, groups to a multiple of 4]."""
    m, k = x.shape
    kp = _up(k, 128)
    x = torch.nn.functional.pad(x.float(), (0, kp - k)).view(m, kp // 128, 128)
    b = _exponents(_finite_abs(x).amax(-1))
    codes = (x * _pow2(254 - b)[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(m, kp)
    exps = torch.nn.functional.pad(b, (0, _up(kp // 128, 4) - kp // 128)).to(torch.uint8)
    return codes, exps


def _dequant(codes, exps, k):
    m, kp = codes.shape
    v = codes.view(torch.float8_e4m3fn).float().view(m, kp // 128, 128) * _pow2(exps[:, : kp // 128])[:, :, None]
    return v.view(m, kp)[:, :k]


def _quant_weight(w):
    """W in 8 bits with one exponent for each 128 x 128 block: codes uint8 [n, k], biased exponents [n blocks, k blocks]."""
    n, k = w.shape
    np_, kp = _up(n, 128), _up(k, 128)
    w = torch.nn.functional.pad(w, (0, kp - k, 0, np_ - n)).view(np_ // 128, 128, kp // 128, 128)
    b = _exponents(_finite_abs(w).amax((1, 3)).contiguous())
    codes = (w * _pow2(254 - b)[:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(np_, kp)
    return codes[:n, :k].contiguous(), b


def _weight_tiles(codes):
    """Rows of codes as the library keeps weights: tiles of 16 rows and 128 columns, zeros past the ends,
    [rows/16][columns/128][2 halves][4 column blocks of 32][16 rows][16 bytes]."""
    n, k = codes.shape
    np_, kp = _up(n, 16), _up(k, 128)
    c = torch.nn.functional.pad(codes, (0, kp - k, 0, np_ - n))
    return c.view(np_ // 16, 16, kp // 128, 4, 2, 16).permute(0, 2, 4, 3, 1, 5).contiguous()


def _weight_exps(b):
    return torch.nn.functional.pad(b, (0, _up(b.shape[1], 4) - b.shape[1])).to(torch.uint8).contiguous()


def _pattern(g, n, k):
    """A 2:4 pattern: the kept positions' columns [n, k/2] and the same as index words (uint8 [n, k/8])."""
    first = torch.randint(0, 6, (n, k // 4), device="cuda", generator=g)
    lo = torch.tensor([0, 0, 0, 1, 1, 2], device="cuda")[first]
    hi = torch.tensor([1, 2, 3, 2, 3, 3], device="cuda")[first]
    nib = (lo | hi << 2).view(n, k // 8, 2)
    meta = (nib[:, :, 0] | nib[:, :, 1] << 4).to(torch.uint8)
    at = torch.stack((lo, hi), -1) + 4 * torch.arange(k // 4, device="cuda")[None, :, None]
    return at.view(n, k // 2), meta


def prepare(case, seed):
    g = _gen(seed)
    kind, m, k = case["kind"], case["m"], case["k"]
    dt = DT[case["dtype"]]
    s = {"case": case}
    if kind in ("norm", "norm_bwd"):
        pt = DT[case["params"]]
        x = _act(g, m, k).to(dt)
        s["gamma"] = (1.0 + _normal(g, (k,), 0.2)).to(pt)
        s["beta"] = None if case["rms"] else _normal(g, (k,), 0.2).to(pt)
        s["x"] = x
        if kind == "norm_bwd":
            s["dy"] = _normal(g, (m, k), 1e-2).to(dt)
            # the forward's statistics, in fp32 as it leaves them
            xd = x.double()
            mean = torch.zeros(m, 1, device="cuda", dtype=torch.float64) if case["rms"] else xd.mean(-1, keepdim=True)
            s["rstd"] = ((xd - mean).square().mean(-1) + EPS).rsqrt().float()
            s["mean"] = None if case["rms"] else mean[:, 0].float()
            if case["q8"]:
                codes, exps = _quant(x)
                s["x"] = {"codes": codes, "exps": exps, "M": m, "K": k}
    elif kind == "ckpt":
        s["x"] = _act(g, m, k).to(dt)
    elif kind == "linear":
        n = case["n"]
        rows = _normal(g, (m, n), 1e-2) if case["dx"] else _act(g, m, k)
        s["x"] = rows.to(dt)
        codes, b = _quant_weight(_normal(g, (n, k), 0.02))
        if case["dx"]:       # the transposed pack: rows k, reduction n
            codes, b = codes.t().contiguous(), b.t().contiguous()
            s["p"] = {"codesT": _weight_tiles(codes), "expsT": _weight_exps(b), "N": n, "K": k}
        else:
            s["p"] = {"codes": _weight_tiles(codes), "exps": _weight_exps(b), "N": n, "K": k}
        s["rows"], s["blocks"] = codes, b      # the same weight row by row
    elif kind == "grad_w":
        n = case["n"]
        s["dy"] = _normal(g, (m, n), 1e-2).to(dt)
        codes, exps = _quant(_act(g, m, k).to(dt))
        s["x"] = {"codes": codes, "exps": exps, "M": m, "K": k}
        if case["mask"]:
            s["at"], meta = _pattern(g, n, k)
            s["p"] = {"meta": meta, "N": n, "K": k}
    return s


# --------------------------------------------------------------------------------- the plain form
def _weight(s):
    rows, b = s["rows"], s["blocks"]
    n, k = rows.shape
    scale = _pow2(b).repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    return rows.view(torch.float8_e4m3fn).float() * scale


def _plain(s):
    case = s["case"]
    kind, k, dt = case["kind"], case["k"], DT[case["dtype"]]
    if kind == "norm":
        x = s["x"].float()
        mean = None if case["rms"] else x.mean(-1, keepdim=True)
        c = x if mean is None else x - mean
        rstd = (c.square().mean(-1, keepdim=True) + EPS).rsqrt()
        y = c * rstd * s["gamma"].float()
        if s["beta"] is not None:
            y = y + s["beta"].float()
        if case["q8"]:
            y = _dequant(*_quant(y), k)
        return [y.to(dt), rstd[:, 0]] + ([] if mean is None else [mean[:, 0]])
    if kind == "norm_bwd":
        x = _dequant(s["x"]["codes"], s["x"]["exps"], k) if case["q8"] else s["x"].float()
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xhat = (x if case["rms"] else x - s["mean"][:, None]) * rstd
        t = dy * s["gamma"].float()
        dx = t - xhat * (t * xhat).mean(-1, keepdim=True)
        if not case["rms"]:
            dx = dx - t.mean(-1, keepdim=True)
        return [(dx * rstd).to(dt), (dy * xhat).sum(0)] + ([] if case["rms"] else [dy.sum(0)])
    if kind == "ckpt":
        return _dequant(*_quant(s["x"]), k).to(dt)
    if kind == "linear":
        x = s["x"]
        return (_dequant(*_quant(x), x.shape[1]) @ _weight(s).t()).to(DT[case["out"]])
    dw = s["dy"].float().t() @ _dequant(s["x"]["codes"], s["x"]["exps"], k)
    return dw.gather(1, s["at"]) if case["mask"] else dw


def run(s):
    if not own:
        return _plain(s)
    from paper_2608_24070_amd import slim
    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        y, mean, rstd = slim.norm(s["x"], s["gamma"], s["beta"], eps=EPS, rms=case["rms"], q8=case["q8"])
        if case["q8"]:
            y = slim.dequant8(y, DT[case["dtype"]])
        return [y, rstd] + ([] if mean is None else [mean])
    if kind == "norm_bwd":
        dx, dgamma, dbeta = slim.norm_bwd(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"])
        return [dx, dgamma] + ([] if dbeta is None else [dbeta])
    if kind == "ckpt":
        return slim.dequant8(slim.quant8(s["x"]), DT[case["dtype"]])
    if kind == "linear":
        if case["dx"]:
            return slim.bwd_dx8(s["x"], s["p"], dtype=DT[case["out"]])
        return slim.linear8(s["x"], s["p"], dtype=DT[case["out"]])
    return slim.grad_w8(s["dy"], s["x"], s["p"] if case["mask"] else None)


# --------------------------------------------------------------------------------- 64 bits
def _quant64(x, dims):
    """Values of x [.., groups' axes ..] after their rounding to 8 bits, from the definition, in 64 bits; `dims` span a group."""
    a = _finite_abs(x).amax(dims, keepdim=True)
    f, p = torch.frexp(a / 448.0)
    e = torch.where(f > 0.5, p, p - 1).clamp(min=-126)
    e = torch.where(a > 0, e, torch.full_like(e, -126)).double()
    v = x * torch.exp2(-e)
    step = torch.exp2(torch.frexp(v)[1].double().sub(1).clamp(min=-6) - 3)
    return torch.round(v / step) * step * torch.exp2(e)


def _rows64(x):
    m, k = x.shape
    kp = _up(k, 128)
    x = torch.nn.functional.pad(x.double(), (0, kp - k)).view(m, kp // 128, 128)
    return _quant64(x, (2,)).view(m, kp)[:, :k]


def _codes64(codes):
    """e4m3 codes as 64-bit values: sign, four exponent bits (bias 7), three mantissa bits."""
    c = codes.to(torch.int64)
    e, f = c >> 3 & 15, (c & 7).double()
    mag = torch.where(e > 0, (8 + f) * torch.exp2(e.double() - 10), f * 2.0 ** -9)
    return torch.where(c & 128 > 0, -mag, mag)


def _checkpoint64(q, k):
    m, kp = q["codes"].shape
    e = q["exps"][:, : kp // 128].double() - 127
    return (_codes64(q["codes"]).view(m, kp // 128, 128) * torch.exp2(e)[:, :, None]).view(m, kp)[:, :k]


def exact(case, seed):
    """What ``run`` returns, from the operators' definitions in 64 bits."""
    s = prepare(case, seed)
    kind, k = case["kind"], case["k"]
    if kind == "norm":
        x = s["x"].double()
        mean = 0.0 if case["rms"] else x.sum(1) / k
        d = x if case["rms"] else x - mean[:, None]
        rstd = 1.0 / torch.sqrt((d * d).sum(1) / k + EPS)
        y = d * rstd[:, None] * s["gamma"].double()
        if s["beta"] is not None:
            y = y + s["beta"].double()
        # with q8, y before its rounding to 8 bits: a value within a last fp32 place of a rounding boundary has two right
        # codes, so that rounding is held to the plain form's, and both sides' distance from y is told here
        return [y, rstd] + ([] if case["rms"] else [mean])
    if kind == "norm_bwd":
        x = _checkpoint64(s["x"], k) if case["q8"] else s["x"].double()
        dy, r = s["dy"].double(), s["rstd"].double()[:, None]
        xh = x * r if case["rms"] else (x - s["mean"].double()[:, None]) * r
        t = dy * s["gamma"].double()
        dx = r / k * (k * t - xh * (t * xh).sum(1, keepdim=True) - (0.0 if case["rms"] else t.sum(1, keepdim=True)))
        return [dx, (dy * xh).sum(0)] + ([] if case["rms"] else [dy.sum(0)])
    if kind == "ckpt":
        return _rows64(s["x"])
    if kind == "linear":
        rows, b = s["rows"], s["blocks"].double() - 127
        n, c = rows.shape
        i, j = torch.arange(n, device="cuda") // 128, torch.arange(c, device="cuda") // 128
        w = _codes64(rows) * torch.exp2(b)[i][:, j]
        return torch.matmul(_rows64(s["x"]), w.t())
    dw = torch.matmul(s["dy"].double().t(), _checkpoint64(s["x"], k))
    return torch.gather(dw, 1, s["at"]) if case["mask"] else dw


# --------------------------------------------------------------------------------- necessary work
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


def _q8_bytes(m, k):
    return m * (_up(k, 128) + _up(k, 128) // 128)


def work(case):
    kind, m, k = case["kind"], case["m"], case["k"]
    b = BYTES[case["dtype"]]
    if kind == "norm":
        stats = 4 * m * (1 if case["rms"] else 2)
        par = BYTES[case["params"]] * k * (1 if case["rms"] else 2)
        # the 8-bit result is written, and read and widened again by the restoring call
        out = 2 * _q8_bytes(m, k) + b * m * k if case["q8"] else b * m * k
        return {"bytes": b * m * k + par + stats + out, "flops": 8 * m * k}
    if kind == "norm_bwd":
        stats = 4 * m * (1 if case["rms"] else 2)
        x = _q8_bytes(m, k) if case["q8"] else b * m * k
        return {"bytes": x + 2 * b * m * k + stats + BYTES[case["params"]] * k + 4 * k * (1 if case["rms"] else 2),
                "flops": 14 * m * k}
    if kind == "ckpt":
        return {"bytes": 2 * b * m * k + 2 * _q8_bytes(m, k), "flops": 4 * m * k}
    n = case["n"]
    if kind == "linear":
        red, cols = (n, k) if case["dx"] else (k, n)
        return {"bytes": b * m * red + n * k + _up(n, 128) * _up(k, 128) // 16384 + BYTES[case["out"]] * m * cols,
                "flops": 2 * m * n * k}
    kept = n * k // 2 if case["mask"] else n * k
    return {"bytes": b * m * n + _q8_bytes(m, k) + (n * k // 8 if case["mask"] else 0) + 4 * kept, "flops": 2 * m * n * k}
