"""The MLP operators around the 8-bit products whose speed is followed: a product with bias, activation, gate and residual in its
epilogue, the gradient through an activation (behind an input gradient's product, or by itself), a router, and a whole layer of
experts for a few tokens.

A case is a dict of plain values with a ``kind``:

``act``      y = act(X W^T + bias) * mul + residual for a 16-bit X [m, k], which the call turns into 8 bits, and an 8-bit W [n, k];
             bias, mul and residual where the case has them. ``pre``: the sum before the activation leaves too, for the backward.
             ``q8``: y (and the sum) leave in 8 bits and are returned as the values they stand for, in the case's type
``bwd_act``  with dh = dY W for dY [m, n] (the input gradient of a product), and the kept u = ``pre`` of the product before it
             [m, k], 16 bits or with ``q8`` 8-bit rows: du = dh * mul * act'(u), with ``mul`` also dmul = dh * act(u), with
             ``bias`` also dbias, the sums of du over the rows, in the case's type
``act_bwd``  the same from a dh [m, k] at hand; dbias in fp32
``route``    the k largest of softmax(X Wr^T) over e experts for each row, the lower expert first where two are equal, as expert
             numbers (int32) and weights (fp32), which with ``renorm`` are divided by their sum
``moe``      ``route``, then y[i] = sum_j weight[i, j] down_e(act(gate_e(x_i)) * up_e(x_i)), e = expert[i, j], with 8-bit weights of
             the experts and 16-bit activations (``q8``: x is 8-bit rows as a norm leaves them); ``residual``: y + residual

8-bit values are e4m3 (OCP; 3 mantissa bits, largest 448) with one power of two 2^e for each group of 128 consecutive
values of a row (for weights: for each block of 128 x 128), e the smallest integer >= -126 for which the group's largest
magnitude / 2^e does not pass 448. Values past the last column count as zero.

Activations: relu, gelu x Phi(x), gelu_tanh x (1 + tanh(sqrt(2 / pi) (x + 0.044715 x^3))) / 2, silu x / (1 + exp(-x)), none.
"""
import math

import torch

own = False     # False: the plain form (elementary torch operations in 32 bits); True: the library's entry points

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # one user's decoding step at a 7B block's gate projection, with the up projection's result as the gate's factor: the
        # smallest product, all latency
        {"name": "act_1", "kind": "act", "m": 1, "n": 11008, "k": 4096, "dtype": "bf16", "act": "silu", "bias": False,
         "mul": True, "residual": False, "pre": False, "q8": False},
        # a ragged batch of 45 decoding on a 13B MLP's first product: its result is the second product's 8-bit operand
        {"name": "act_45", "kind": "act", "m": 45, "n": 13824, "k": 5120, "dtype": "fp16", "act": "gelu", "bias": True,
         "mul": False, "residual": False, "pre": False, "q8": True},
        # a training batch on the 70B MLP's first product: the activation and its argument are kept in 8 bits
        {"name": "act_4096", "kind": "act", "m": 4096, "n": 28672, "k": 8192, "dtype": "bf16", "act": "gelu_tanh", "bias": True,
         "mul": False, "residual": False, "pre": True, "q8": True},
        # a small model's backward over a few odd sequences
        {"name": "bwd_act_333", "kind": "bwd_act", "m": 333, "n": 768, "k": 2051, "dtype": "fp16", "act": "gelu", "bias": True,
         "mul": False, "q8": False},
        # the 70B gated MLP's backward over a training batch, from 8-bit checkpoints
        {"name": "bwd_act_4096", "kind": "bwd_act", "m": 4096, "n": 8192, "k": 28672, "dtype": "bf16", "act": "silu",
         "bias": False, "mul": True, "q8": True},
        # an odd activation's gradient by itself: rows that end inside a group and start off alignment
        {"name": "act_bwd_100", "kind": "act_bwd", "m": 100, "k": 4097, "dtype": "fp16", "act": "gelu", "bias": True, "mul": False,
         "q8": False},
        # the 70B MLP's widest activation over a training batch, its argument kept in 8 bits
        {"name": "act_bwd_8192", "kind": "act_bwd", "m": 8192, "k": 28672, "dtype": "bf16", "act": "gelu_tanh", "bias": True,
         "mul": False, "q8": True},
        # one user's token to its experts
        {"name": "route_1", "kind": "route", "m": 1, "e": 64, "d": 4096, "top": 8, "dtype": "bf16", "router": "bf16", "renorm": True},
        # a batch of 61 tokens over many experts, the router kept in fp32
        {"name": "route_61", "kind": "route", "m": 61, "e": 250, "d": 8192, "top": 6, "dtype": "fp16", "router": "fp32", "renorm": False},
        # one user's token through a layer of 64 small experts
        {"name": "moe_1", "kind": "moe", "m": 1, "e": 64, "d": 4096, "f": 1024, "top": 8, "dtype": "bf16", "router": "bf16",
         "act": "silu", "renorm": True, "q8": False, "residual": False},
        # seven users on eight experts of a 7B MLP's size
        {"name": "moe_7", "kind": "moe", "m": 7, "e": 8, "d": 4096, "f": 11008, "top": 2, "dtype": "fp16", "router": "fp16",
         "act": "silu", "renorm": True, "q8": False, "residual": True},
        # a batch of 61 on 40 experts of odd width, behind a norm that leaves 8 bits: nearly every expert is read
        {"name": "moe_61", "kind": "moe", "m": 61, "e": 40, "d": 5120, "f": 1700, "top": 4, "dtype": "bf16", "router": "fp32",
         "act": "gelu_tanh", "renorm": False, "q8": True, "residual": True},
    ]


MOST_PRODUCT = 4096 * 28672 * 8192
MOST_VALUES = 8192 * 28672
MOST_EXPERTS = 8 * 4096 * 11008      # values of one of the experts' three weights
MOST_ROWS = 64                       # a few tokens


def _log(rng, lo, hi):
    return lo * (hi / lo) ** rng.random()


def _size(rng, lo, hi):
    """A width over lo .. hi: any number, or a multiple of 16 or 128 as layers mostly have them."""
    v, mult = int(_log(rng, lo, hi)), rng.choice([1, 16, 128, 128])
    return max(mult, v // mult * mult)


ACTS = ["relu", "gelu", "gelu_tanh", "silu"]


def draw(rng):
    """One more case of the listed ranges, no larger than the largest listed one."""
    kind = rng.choice(["act", "act", "act", "bwd_act", "bwd_act", "act_bwd", "act_bwd", "route", "moe", "moe", "moe"])
    dtype, flip = rng.choice(["bf16", "bf16", "fp16"]), lambda p=0.5: rng.random() < p
    if kind in ("route", "moe"):
        m, e, d = int(_log(rng, 1, MOST_ROWS + 1)), int(_log(rng, 4, 257)), _size(rng, 256, 8192)
        case = {"kind": kind, "m": min(m, MOST_ROWS), "e": min(e, 256), "d": d, "top": min(rng.randint(1, 8), e), "dtype": dtype,
                "router": rng.choice([dtype, "fp32"]), "renorm": flip()}
        if kind == "moe":
            f = _size(rng, 256, 11008)
            case.update({"e": max(case["top"], min(case["e"], MOST_EXPERTS // (d * f))), "f": f, "act": rng.choice(["silu", "gelu", "gelu_tanh"]),
                         "q8": flip(0.3), "residual": flip()})
        return case
    k, m = _size(rng, 128, 28672), int(_log(rng, 1, 8193))
    act = rng.choice(ACTS)
    if kind == "act_bwd":
        return {"kind": kind, "m": max(1, min(m, 8192, MOST_VALUES // k)), "k": k, "dtype": dtype, "act": act, "bias": flip(), "mul": flip(),
                "q8": flip()}
    n = _size(rng, 128, 28672)
    case = {"kind": kind, "m": max(1, min(m, 8192, MOST_PRODUCT // (n * k))), "n": n, "k": k, "dtype": dtype, "act": act, "bias": flip(),
            "mul": flip(0.4), "q8": flip()}
    if kind == "act":
        case.update({"act": rng.choice(ACTS + ["none"]), "residual": flip(0.4), "pre": flip(0.4)})
    return case


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


def _rows8(x):
    codes, exps = _quant(x)
    return {"codes": codes, "exps": exps, "M": x.shape[0], "K": x.shape[1]}


def _quant_weight(w):
    """W [.., n, k] in 8 bits with one exponent for each 128 x 128 block: codes uint8 [.., n, k], biased exponents [.., n blocks,
    k blocks]."""
    *e, n, k = w.shape
    np_, kp = _up(n, 128), _up(k, 128)
    w = torch.nn.functional.pad(w, (0, kp - k, 0, np_ - n)).view(-1, np_ // 128, 128, kp // 128, 128)
    b = _exponents(_finite_abs(w).amax((2, 4)).contiguous())
    codes = (w * _pow2(254 - b)[:, :, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(*e, np_, kp)
    return codes[..., :n, :k].contiguous(), b.view(*e, np_ // 128, kp // 128)


def _weight_tiles(codes):
    """Rows of codes as the library keeps weights: tiles of 16 rows and 128 columns, zeros past the ends,
    [..][rows/16][columns/128][2 halves][4 column blocks of 32][16 rows][16 bytes]."""
    *e, n, k = codes.shape
    np_, kp = _up(n, 16), _up(k, 128)
    c = torch.nn.functional.pad(codes, (0, kp - k, 0, np_ - n)).view(-1, np_ // 16, 16, kp // 128, 4, 2, 16)
    return c.permute(0, 1, 3, 5, 4, 2, 6).contiguous().view(*e, np_ // 16, kp // 128, 2, 4, 16, 16)


def _weight_exps(b):
    return torch.nn.functional.pad(b, (0, _up(b.shape[-1], 4) - b.shape[-1])).to(torch.uint8).contiguous()


def _experts(g, e, n, k):
    """An 8-bit weight for each of e experts: as the library keeps them, and row by row."""
    codes, b = _quant_weight(_normal(g, (e, n, k), 0.02))
    return {"codes": _weight_tiles(codes), "exps": _weight_exps(b), "E": e, "N": n, "K": k}, (codes, b)


def prepare(case, seed):
    g = _gen(seed)
    kind, m, dt = case["kind"], case["m"], DT[case["dtype"]]
    s = {"case": case}
    if kind in ("act", "bwd_act"):
        n, k = case["n"], case["k"]
        codes, b = _quant_weight(_normal(g, (n, k), 0.02))
        if kind == "act":
            s["x"] = _act(g, m, k).to(dt)
            s["p"] = {"codes": _weight_tiles(codes), "exps": _weight_exps(b), "N": n, "K": k}
            s["bias"] = _normal(g, (n,), 0.5) if case["bias"] else None
            s["mul"] = _normal(g, (m, n), 1.0).to(dt) if case["mul"] else None
            s["residual"] = _act(g, m, n).to(dt) if case["residual"] else None
        else:                # the transposed pack: rows k, reduction n
            s["dy"] = _normal(g, (m, n), 1e-2).to(dt)
            codes, b = codes.t().contiguous(), b.t().contiguous()
            s["p"] = {"codesT": _weight_tiles(codes), "expsT": _weight_exps(b), "N": n, "K": k}
        s["rows"], s["blocks"] = codes, b      # the same weight row by row
    if kind in ("bwd_act", "act_bwd"):
        k = case["k"]
        keep = _rows8 if case["q8"] else (lambda v: v)
        s["u"] = keep(_normal(g, (m, k), 1.5).to(dt))
        s["mul"] = keep(_normal(g, (m, k), 1.0).to(dt)) if case["mul"] else None
        if kind == "act_bwd":
            s["dh"] = _normal(g, (m, k), 1e-2).to(dt)
    if kind in ("route", "moe"):
        e, d = case["e"], case["d"]
        x = _act(g, m, d).to(dt)
        s["x"] = _rows8(x) if case.get("q8") else x
        # logits of order one: they are what spreads tokens over experts
        s["router"] = (_normal(g, (e, d), 0.5 * d ** -0.5)).to(DT[case["router"]])
    if kind == "moe":
        f = case["f"]
        s["gate"], s["gate_rows"] = _experts(g, e, f, d)
        s["up"], s["up_rows"] = _experts(g, e, f, d)
        s["down"], s["down_rows"] = _experts(g, e, d, f)
        s["residual"] = _act(g, m, d).to(dt) if case["residual"] else None
    return s


# --------------------------------------------------------------------------------- the plain form
def _value(act, u):
    if act == "relu":
        return torch.where(u < 0, torch.zeros_like(u), u)
    if act == "gelu":
        return 0.5 * u * torch.erfc(u * -(0.5 ** 0.5))
    if act == "gelu_tanh":
        return u / (1 + torch.exp(-2 * (2 / math.pi) ** 0.5 * (u + 0.044715 * u * u * u)))
    if act == "silu":
        return u / (1 + torch.exp(-u))
    return u


def _slope(act, u):
    if act == "relu":
        return (u > 0).float()
    if act == "gelu":
        return 0.5 * torch.erfc(u * -(0.5 ** 0.5)) + u * torch.exp(-0.5 * u * u) * (2 * math.pi) ** -0.5
    if act == "gelu_tanh":
        c = 2 * (2 / math.pi) ** 0.5
        p = 1 / (1 + torch.exp(-c * (u + 0.044715 * u * u * u)))
        return p + u * p * (1 - p) * c * (1 + 3 * 0.044715 * u * u)
    p = 1 / (1 + torch.exp(-u))
    return p + u * p * (1 - p)


def _wide(codes, b):
    """A weight's values [.., n, k] in fp32 from its codes row by row and its blocks' exponents."""
    n, k = codes.shape[-2:]
    scale = _pow2(b).repeat_interleave(128, -2)[..., :n, :].repeat_interleave(128, -1)[..., :k]
    return codes.view(torch.float8_e4m3fn).float() * scale


def _kept(v, case):
    return _dequant(v["codes"], v["exps"], case["k"]) if case["q8"] else v.float()


def _moved(s, dh):
    """What `bwd_act` and `act_bwd` return, from dh in fp32."""
    case, dt = s["case"], DT[s["case"]["dtype"]]
    u = _kept(s["u"], case)
    du = dh * _slope(case["act"], u)
    out = []
    if case["mul"]:
        du = du * _kept(s["mul"], case)
        out.append((dh * _value(case["act"], u)).to(dt))
    if case["bias"]:
        out.append(du.sum(0).to(dt if case["kind"] == "bwd_act" else torch.float32))
    return [du.to(dt)] + out


def _routed(s):
    case, x = s["case"], s["x"]
    x = _dequant(x["codes"], x["exps"], case["d"]) if case.get("q8") else x
    # two logits may be as near as their sums' last places in 32 bits
    logits = x.double() @ s["router"].double().t()
    p = torch.exp(logits - logits.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    top, ids = torch.sort(p, dim=1, descending=True, stable=True)
    top, ids = top[:, : case["top"]], ids[:, : case["top"]]
    if case["renorm"]:
        top = top / top.sum(1, keepdim=True)
    return x.float(), ids, top.float()


def _plain(s):
    case = s["case"]
    kind, dt = case["kind"], DT[case["dtype"]]
    if kind == "act":
        x, n = s["x"], case["n"]
        z = _dequant(*_quant(x), case["k"]) @ _wide(s["rows"], s["blocks"]).t()
        if s["bias"] is not None:
            z = z + s["bias"]
        y = _value(case["act"], z)
        if s["mul"] is not None:
            y = y * s["mul"].float()
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return [(_dequant(*_quant(v), n) if case["q8"] else v).to(dt) for v in ([y, z] if case["pre"] else [y])]
    if kind == "bwd_act":
        return _moved(s, _dequant(*_quant(s["dy"]), case["n"]) @ _wide(s["rows"], s["blocks"]).t())
    if kind == "act_bwd":
        return _moved(s, s["dh"].float())
    x, ids, weights = _routed(s)
    if kind == "route":
        return [ids.to(torch.int32), weights]
    m, e, d, f, top = (case[v] for v in ("m", "e", "d", "f", "top"))
    if m * top <= e:         # the experts that were picked, each as often as it was
        at = ids.reshape(-1)
        gate, up, down = (_wide(c[at], b[at]) for c, b in (s["gate_rows"], s["up_rows"], s["down_rows"]))
        pairs = x.repeat_interleave(top, 0)[:, :, None]
        h = _value(case["act"], torch.matmul(gate, pairs)) * torch.matmul(up, pairs)
        y = (torch.matmul(down, h)[:, :, 0] * weights.reshape(-1, 1)).view(m, top, d).sum(1)
    else:                    # all experts, with weight zero where they were not picked
        gate, up, down = (_wide(*s[v]) for v in ("gate_rows", "up_rows", "down_rows"))
        h = _value(case["act"], x @ gate.view(e * f, d).t()) * (x @ up.view(e * f, d).t())
        share = torch.zeros((m, e), device=x.device).scatter_(1, ids, weights)
        y = (h.view(m, e, f) * share[:, :, None]).view(m, e * f) @ down.transpose(1, 2).reshape(e * f, d)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return [y.to(dt), ids.to(torch.int32), weights]


def run(s):
    if not own:
        return _plain(s)
    from paper_2608_24070_amd import slim
    case = s["case"]
    kind, dt = case["kind"], DT[case["dtype"]]
    if kind == "act":
        out = slim.linear8_act(s["x"], s["p"], act=case["act"], bias=s["bias"], mul=s["mul"], residual=s["residual"], pre=case["pre"],
                               q8=case["q8"], dtype=dt)
        out = list(out) if case["pre"] else [out]
        return [slim.dequant8(v, dt) for v in out] if case["q8"] else out
    if kind in ("bwd_act", "act_bwd"):
        if kind == "bwd_act":
            du, dmul, dbias = slim.bwd_dx8_act(s["dy"], s["p"], s["u"], act=case["act"], mul=s["mul"], bias=case["bias"], dtype=dt)
        else:
            du, dmul, dbias = slim.act_bwd(s["dh"], s["u"], act=case["act"], mul=s["mul"], bias=case["bias"])
        return [v for v in (du, dmul, dbias) if v is not None]
    ids, weights = slim.route(s["x"], s["router"], case["top"], renorm=case["renorm"])
    if kind == "route":
        return [ids, weights]
    y = slim.moe8(s["x"], s["gate"], s["up"], s["down"], ids, weights, act=case["act"], residual=s["residual"], dtype=dt)
    return [y, ids, weights]


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


def _weight64(codes, b):
    n, c = codes.shape
    i, j = torch.arange(n, device="cuda") // 128, torch.arange(c, device="cuda") // 128
    return _codes64(codes) * torch.exp2(b.double() - 127)[i][:, j]


def _pair64(act, z):
    """act(z) and its derivative from their definitions."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * torch.sigmoid(-z))
    if act == "gelu":
        phi = torch.special.ndtr(z)
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z ** 3))
    return z / 2 * (1 + t), (1 + t) / 2 + z / 2 * (1 - t * t) * c * (1 + 0.134145 * z * z)


def exact(case, seed):
    """What ``run`` returns, from the operators' definitions in 64 bits."""
    kind = case["kind"]
    if kind in ("act", "bwd_act") and case["m"] * case["n"] * case["k"] > MOST_PRODUCT // 4:
        return None          # a product that takes long in 64 bits
    if kind == "act" and case["q8"]:
        return None          # a value near a border of two codes has two right ones: its rounding is held to the plain form's
    s = prepare(case, seed)
    if kind == "act":
        z = torch.matmul(_rows64(s["x"]), _weight64(s["rows"], s["blocks"]).t())
        if case["bias"]:
            z = z + s["bias"].double()
        y = _pair64(case["act"], z)[0]
        if case["mul"]:
            y = y * s["mul"].double()
        if case["residual"]:
            y = y + s["residual"].double()
        return [y, z] if case["pre"] else [y]
    if kind in ("bwd_act", "act_bwd"):
        read = (lambda v: _checkpoint64(v, case["k"])) if case["q8"] else (lambda v: v.double())
        dh = torch.matmul(_rows64(s["dy"]), _weight64(s["rows"], s["blocks"]).t()) if kind == "bwd_act" else s["dh"].double()
        value, slope = _pair64(case["act"], read(s["u"]))
        du = dh * slope
        if case["mul"]:
            du = du * read(s["mul"])
        return [du] + ([dh * value] if case["mul"] else []) + ([du.sum(0)] if case["bias"] else [])
    x = _checkpoint64(s["x"], case["d"]) if case.get("q8") else s["x"].double()
    p = torch.softmax(torch.matmul(x, s["router"].double().t()), 1)
    m, e, top = case["m"], case["e"], case["top"]
    left, ids = p.clone(), torch.zeros((m, top), dtype=torch.int64, device="cuda")
    rows = torch.arange(m, device="cuda")
    for j in range(top):     # the largest that is left, the first of equal ones
        ids[:, j] = (left == left.amax(1, keepdim=True)).to(torch.int8).argmax(1)
        left[rows, ids[:, j]] = -1.0
    weights = torch.gather(p, 1, ids)
    if case["renorm"]:
        weights = weights / weights.sum(1, keepdim=True)
    if kind == "route":
        return [ids.to(torch.int32), weights]
    y = torch.zeros((m, case["d"]), dtype=torch.float64, device="cuda")
    for i in range(e):
        mine = ids == i
        at = mine.any(1).nonzero()[:, 0]
        if not len(at):
            continue
        gate, up, down = (_weight64(c[i], b[i]) for c, b in (s["gate_rows"], s["up_rows"], s["down_rows"]))
        h = _pair64(case["act"], torch.matmul(x[at], gate.t()))[0] * torch.matmul(x[at], up.t())
        y[at] += torch.matmul(h, down.t()) * (weights * mine).sum(1)[at, None]
    if case["residual"]:
        y = y + s["residual"].double()
    return [y, ids.to(torch.int32), weights]


# --------------------------------------------------------------------------------- necessary work
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


def _q8_bytes(m, k):
    return m * (_up(k, 128) + _up(k, 128) // 128)


def work(case):
    kind, m = case["kind"], case["m"]
    b = BYTES[case["dtype"]]
    if kind == "act":
        n, k = case["n"], case["k"]
        # an 8-bit result is written, and read and widened again by the restoring call
        out = (2 * _q8_bytes(m, n) + b * m * n if case["q8"] else b * m * n) * (2 if case["pre"] else 1)
        read = b * m * n * ((1 if case["mul"] else 0) + (1 if case["residual"] else 0)) + (4 * n if case["bias"] else 0)
        return {"bytes": b * m * k + n * k + _up(n, 128) * _up(k, 128) // 16384 + read + out, "flops": 2 * m * n * k}
    if kind in ("bwd_act", "act_bwd"):
        k, two = case["k"], 2 if case["mul"] else 1
        kept = (_q8_bytes(m, k) if case["q8"] else b * m * k) * two
        moved = kept + b * m * k * two + ((b if kind == "bwd_act" else 4) * k if case["bias"] else 0)
        if kind == "act_bwd":
            return {"bytes": b * m * k + moved, "flops": 20 * m * k}
        n = case["n"]
        return {"bytes": b * m * n + n * k + _up(n, 128) * _up(k, 128) // 16384 + moved, "flops": 2 * m * n * k}
    e, d, top = case["e"], case["d"], case["top"]
    x = _q8_bytes(m, d) if case.get("q8") else b * m * d
    routing = {"bytes": x + BYTES[case["router"]] * e * d + 8 * m * top, "flops": 2 * m * e * d}
    if kind == "route":
        return routing
    f = case["f"]
    picked = e * (1 - (1 - top / e) ** m)       # experts that m rows of `top` each reach, on average
    return {"bytes": int(routing["bytes"] + 3 * picked * f * d + b * m * d * (2 if case["residual"] else 1)),
            "flops": routing["flops"] + 6 * m * top * f * d}
