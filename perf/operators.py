"""The operators of a pre-norm residual block, as cases that can be timed and compared.

    h, s = rmsnorm(x + s)          a = act(h W1^T + b1)          s' = a W2^T + b2 + s

for one network or for a population of them ("groups", each with weights of its own): the norm with
the residual's addition, in bf16, fp32 or 8 bits with a scale per row ("norm"), its backward pass
("norm_bwd"), rows quantised to 8 bits ("quant"), the product with bias, activation and residual in
bf16 or over 8-bit operands ("linear"), and the product's backward pass ("linear_bwd").
"""

import math

import torch

own = False  # False: the plain form below; True: the framework's operators

F32, F64, BF16, E4M3 = torch.float32, torch.float64, torch.bfloat16, torch.float8_e4m3fn
E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -126
EPS = 1e-6
SLOPE = 0.2


# ---- cases ------------------------------------------------------------------------------------
def _norm(name, rows, dim, groups=1, type="bf16", residual=True, e4m3=False, keep=False):
    return _named(name, dict(op="norm", groups=groups, rows=rows, dim=dim, type=type,
                             residual=residual, e4m3=e4m3, keep=keep))


def _norm_bwd(name, rows, dim, groups=1, type="bf16", dsum=True):
    return _named(name, dict(op="norm_bwd", groups=groups, rows=rows, dim=dim, type=type, dsum=dsum))


def _quant(name, rows, dim, groups=1, type="bf16"):
    return _named(name, dict(op="quant", groups=groups, rows=rows, dim=dim, type=type))


def _linear(name, rows, k, n, groups=1, type="bf16", act="none", bias=True, residual=False,
            keep=False, out="bf16"):
    return _named(name, dict(op="linear", groups=groups, rows=rows, k=k, n=n, type=type, act=act,
                             bias=bias, residual=residual, keep=keep, out=out))


def _linear_bwd(name, rows, k, n, groups=1, act="none"):
    return _named(name, dict(op="linear_bwd", groups=groups, rows=rows, k=k, n=n, act=act))


def _named(name, case):
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one sample through a served network: its norm, in the 8 bits that the next product reads
        _norm("norm_1x4096_e4m3", 1, 4096, e4m3=True),
        # a large batch through a wide served network
        _norm("norm_16384x8192_e4m3", 16384, 8192, e4m3=True),
        # every cell of a 12x12 grid trains its block: batch 100, hidden width 256
        _norm_bwd("norm_bwd_144x100x256", 100, 256, groups=144),
        # one wide network in training
        _norm_bwd("norm_bwd_8192x4096", 8192, 4096),
        # the batch and width of a small ragged network, between its two products
        _quant("quant_37x500", 37, 500),
        # the hidden activations of a large batch
        _quant("quant_16384x4096", 16384, 4096),
        # one sample through a product: the weights' way through memory
        _linear("linear_1x4096x4096", 1, 4096, 4096, act="silu", residual=True),
        # the output layer of every generator of a 12x12 grid over its five batches of 100
        _linear("linear_144x500x256x784", 500, 256, 784, groups=144, act="tanh"),
        # 8-bit operands whose rows are not whole 16-byte units
        _linear("linear_e4m3_37x1000x500", 37, 1000, 500, type="e4m3", act="relu"),
        # a wide served network, a large batch
        _linear("linear_e4m3_8192x4096x8192", 8192, 4096, 8192, type="e4m3", act="gelu",
                residual=True),
        # sizes that fill no tile, in training
        _linear_bwd("linear_bwd_777x500x1001", 777, 500, 1001, act="lrelu"),
        # a wide network in training
        _linear_bwd("linear_bwd_8192x4096x4096", 8192, 4096, 4096, act="silu"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: a power of two or the repository's 784, an odd number of 8s, or an odd number."""
    v, kind = _log(rng, lo, hi), rng.random()
    if kind < 0.5:
        return max([w for w in (16, 64, 128, 256, 512, 784, 1024, 2048, 4096, 8192) if w <= v])
    return (v // 8 | 1) * 8 if kind < 0.75 and v < hi else min(v | 1, hi - 1)


def _rows(rng, hi):
    """Rows: few of them as likely as many, odd where they are many."""
    v = _log(rng, 1, hi)
    return v | 1 if v > 256 else v


def draw(rng):
    """One more call of the same kinds, over the ranges that the listed ones stand for."""
    op = rng.choice(["norm", "norm_bwd", "quant", "linear", "linear", "linear_e4m3", "linear_bwd"])
    groups = rng.choice([1, 1, 1, _log(rng, 2, 144)])
    if op in ("norm", "norm_bwd", "quant"):
        dim, rows, kind = _width(rng, 64, 8192), _rows(rng, 16384), rng.choice(["bf16", "bf16", "fp32"])
        rows = max(1, min(rows, (1 << 26) // (groups * dim)))
        if op == "quant":
            return _quant(None, rows, dim, groups, kind)
        if op == "norm_bwd":
            return _norm_bwd(None, rows, dim, groups, kind, rng.random() < 0.7)
        return _norm(None, rows, dim, groups, kind, rng.random() < 0.7, rng.random() < 0.4,
                     rng.random() < 0.4)
    k, n, rows = _width(rng, 64, 8192), _width(rng, 16, 8192), _rows(rng, 8192)
    act = rng.choice(["none", "relu", "lrelu", "tanh", "gelu", "silu"])
    rows = max(1, min(rows, (1 << 36) // (groups * k * n)))
    while groups * n * k > 1 << 27:
        groups = groups // 2
    if op == "linear_bwd":
        return _linear_bwd(None, rows, k, n, groups, act)
    e4m3 = op == "linear_e4m3"
    return _linear(None, rows, k, n, groups, "e4m3" if e4m3 else "bf16", act, rng.random() < 0.7,
                   rng.random() < 0.5, rng.random() < 0.4,
                   "fp32" if not e4m3 and rng.random() < 0.2 else "bf16")


_TYPES = {"bf16": BF16, "fp32": F32, "e4m3": E4M3}
_BYTES = {"bf16": 2, "fp32": 4, "e4m3": 1}


def work(case):
    c = case
    g = c["groups"]
    if c["op"] in ("norm", "norm_bwd", "quant"):
        e, rows, b = g * c["rows"] * c["dim"], g * c["rows"], _BYTES[c["type"]]
        if c["op"] == "quant":
            return {"bytes": e * (b + 1) + 4 * rows, "flops": 3 * e}
        if c["op"] == "norm":
            moved = e * (b * (1 + 2 * c["residual"]) + (1 if c["e4m3"] else b))
            moved += 4 * g * c["dim"] + 4 * rows * (c["e4m3"] + c["keep"])
            return {"bytes": moved, "flops": 6 * e}
        return {"bytes": e * b * (3 + c["dsum"]) + 4 * rows + 8 * g * c["dim"], "flops": 10 * e}
    m, n, k = c["rows"], c["n"], c["k"]
    if c["op"] == "linear":
        b, o = _BYTES[c["type"]], _BYTES[c["out"]]
        moved = g * ((m + n) * k * b + m * n * (o * (1 + c["residual"]) + 2 * c["keep"]))
        moved += g * 4 * (n * c["bias"] + ((m + n) if c["type"] == "e4m3" else 0))
        return {"bytes": moved, "flops": 2 * g * m * n * k}
    moved = g * 2 * (m * n * (1 + (c["act"] != "none")) + 2 * m * k + 2 * n * k) + 4 * g * n
    return {"bytes": moved, "flops": 4 * g * m * n * k}


# ---- inputs -----------------------------------------------------------------------------------
def _randn(gen, shape, std, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=F32).mul_(std).to(dtype)


def _rows_to_e4m3(x):
    """x in 8 bits with a scale per row, as a served network's weights and inputs are held."""
    scale = (x.float().abs().amax(dim=-1) / E4M3_MAX).clamp_(min=SCALE_MIN)
    return (x.float() / scale[..., None]).to(E4M3), scale


def _shape(case, *dims):
    return dims if case["groups"] == 1 else (case["groups"],) + dims


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    c, s = case, {"case": case}
    if c["op"] in ("norm", "norm_bwd", "quant"):
        t, rows, dim = _TYPES[c["type"]], c["rows"], c["dim"]
        s["x"] = _randn(gen, _shape(c, rows, dim), 1.0, t)
        if c["op"] == "quant":
            return s
        s["weight"] = 1.0 + _randn(gen, _shape(c, dim), 0.1, F32)
        if c["op"] == "norm":
            s["residual"] = _randn(gen, _shape(c, rows, dim), 2.0, t) if c["residual"] else None
            return s
        s["rstd"] = 1.0 / torch.sqrt(s["x"].float().square().mean(dim=-1) + EPS)
        s["dy"] = _randn(gen, _shape(c, rows, dim), 0.01, t)
        s["dsum"] = _randn(gen, _shape(c, rows, dim), 0.01, t) if c["dsum"] else None
        return s
    m, n, k = c["rows"], c["n"], c["k"]
    x, w = (_randn(gen, _shape(c, m, k), 1.0, BF16), _randn(gen, _shape(c, n, k), k ** -0.5, BF16))
    if c["op"] == "linear":
        s["bias"] = _randn(gen, _shape(c, n), 0.1, F32) if c["bias"] else None
        s["residual"] = (_randn(gen, _shape(c, m, n), 1.0, _TYPES[c["out"]]) if c["residual"]
                         else None)
        if c["type"] == "e4m3":
            (s["x"], s["x_scale"]), (s["w"], s["w_scale"]) = _rows_to_e4m3(x), _rows_to_e4m3(w)
        else:
            s["x"], s["w"], s["x_scale"], s["w_scale"] = x, w, None, None
        return s
    s["x"], s["w"] = x, w
    s["dy"] = _randn(gen, _shape(c, m, n), 0.01, BF16)
    s["pre"] = _randn(gen, _shape(c, m, n), 1.0, BF16) if c["act"] != "none" else None
    return s


# ---- the plain forms, in 32 bits ----------------------------------------------------------------
def _act(act, u):
    if act == "relu":
        return torch.where(u > 0, u, torch.zeros_like(u))
    if act == "lrelu":
        return torch.where(u > 0, u, SLOPE * u)
    if act == "tanh":
        return torch.tanh(u)
    if act == "gelu":
        return 0.5 * u * (1 + torch.tanh(math.sqrt(2 / math.pi) * (u + 0.044715 * u * u * u)))
    if act == "silu":
        return u / (1 + torch.exp(-u))
    return u


def _act_slope(act, u):
    """The activation's derivative at u."""
    if act == "relu":
        return (u > 0).to(u.dtype)
    if act == "lrelu":
        return torch.where(u > 0, torch.ones_like(u), torch.full_like(u, SLOPE))
    if act == "tanh":
        t = torch.tanh(u)
        return 1 - t * t
    if act == "gelu":
        a = math.sqrt(2 / math.pi)
        t = torch.tanh(a * (u + 0.044715 * u * u * u))
        return 0.5 * (1 + t) + 0.5 * u * (1 - t * t) * a * (1 + 3 * 0.044715 * u * u)
    s = 1 / (1 + torch.exp(-u))
    return s * (1 + u * (1 - s))


def _plain(s):
    c = s["case"]
    if c["op"] == "norm":
        total = s["x"].float()
        if c["residual"]:
            total = total + s["residual"].float()
        rstd = 1.0 / torch.sqrt((total * total).mean(dim=-1) + EPS)
        y = total * rstd[..., None] * s["weight"][..., None, :]
        out = {}
        if c["e4m3"]:
            out["scale"] = (y.abs().amax(dim=-1) / E4M3_MAX).clamp_(min=SCALE_MIN)
            out["y"] = (y / out["scale"][..., None]).to(E4M3)
        else:
            out["y"] = y.to(_TYPES[c["type"]])
        if c["residual"]:
            out["sum"] = total.to(_TYPES[c["type"]])
        if c["keep"]:
            out["rstd"] = rstd
        return out
    if c["op"] == "norm_bwd":
        x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][..., None]
        g = dy * s["weight"][..., None, :]
        dx = rstd * (g - x * (rstd * rstd * (g * x).mean(dim=-1, keepdim=True)))
        if c["dsum"]:
            dx = dx + s["dsum"].float()
        return {"dx": dx.to(_TYPES[c["type"]]), "dweight": (dy * x * rstd).sum(dim=-2)}
    if c["op"] == "quant":
        q, scale = _rows_to_e4m3(s["x"])
        return {"q": q, "scale": scale}
    if c["op"] == "linear":
        u = s["x"].float() @ s["w"].float().transpose(-1, -2)
        if c["type"] == "e4m3":
            u = u * s["x_scale"][..., None] * s["w_scale"][..., None, :]
        if c["bias"]:
            u = u + s["bias"][..., None, :]
        y = _act(c["act"], u)
        if c["residual"]:
            y = y + s["residual"].float()
        out = {"y": y.to(_TYPES[c["out"]])}
        if c["keep"]:
            out["pre"] = u.to(BF16)
        return out
    du = s["dy"].float()
    if c["act"] != "none":
        du = du * _act_slope(c["act"], s["pre"].float())
    return {"dx": (du @ s["w"].float()).to(BF16),
            "dw": (du.transpose(-1, -2) @ s["x"].float()).to(BF16), "db": du.sum(dim=-2)}


# ---- the framework's operators -------------------------------------------------------------------
def _own(s):
    from paper_1811_12843_gb300 import operators as ops
    c = s["case"]
    if c["op"] == "norm":
        r = ops.rmsnorm(s["x"], s["weight"], residual=s["residual"], eps=EPS, e4m3=c["e4m3"],
                        keep=c["keep"])
        out = {"y": r.y}
        if c["e4m3"]:
            out["scale"] = r.scale
        if c["residual"]:
            out["sum"] = r.sum
        if c["keep"]:
            out["rstd"] = r.rstd
        return out
    if c["op"] == "norm_bwd":
        dx, dweight = ops.rmsnorm_backward(s["dy"], s["x"], s["rstd"], s["weight"], dsum=s["dsum"])
        return {"dx": dx, "dweight": dweight}
    if c["op"] == "quant":
        q, scale = ops.quantize_rows(s["x"])
        return {"q": q, "scale": scale}
    if c["op"] == "linear":
        y, pre = ops.linear(s["x"], s["w"], s["bias"], act=c["act"], slope=SLOPE,
                            residual=s["residual"], x_scale=s["x_scale"], w_scale=s["w_scale"],
                            out_dtype=_TYPES[c["out"]], keep=c["keep"])
        return {"y": y, "pre": pre} if c["keep"] else {"y": y}
    dx, dw, db = ops.linear_backward(s["dy"], s["x"], s["w"], act=c["act"], slope=SLOPE, pre=s["pre"])
    return {"dx": dx, "dw": dw, "db": db}


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definitions, in 64 bits -------------------------------------------------------------------
def _sigmoid64(v):
    """1 / (1 + e^-v) without overflow."""
    e = torch.exp(-v.abs())
    return torch.where(v >= 0, torch.ones_like(e), e) / (1 + e)


def _exact_act(act, u):
    """(act(u), act'(u)): gelu is u times the logistic function of 2 sqrt(2/pi) (u + 0.044715 u^3)."""
    one, zero = torch.ones_like(u), torch.zeros_like(u)
    if act == "relu":
        return torch.maximum(u, zero), torch.where(u > 0, one, zero)
    if act == "lrelu":
        m = torch.where(u > 0, one, SLOPE * one)
        return u * m, m
    if act == "tanh":
        t = 2 * _sigmoid64(2 * u) - 1
        return t, (1 - t) * (1 + t)
    if act in ("gelu", "silu"):
        c1, c3 = ((2 * math.sqrt(2 / math.pi), 2 * math.sqrt(2 / math.pi) * 0.044715)
                  if act == "gelu" else (1.0, 0.0))
        g = _sigmoid64(c1 * u + c3 * u ** 3)
        return u * g, g + u * g * (1 - g) * (c1 + 3 * c3 * u ** 2)
    return u, one


def exact(case, seed):
    """What run() returns before its one rounding to the output's type (8-bit values: the row over
    its scale)."""
    s, c = prepare(case, seed), case
    d = {k: v.to(F64) for k, v in s.items() if isinstance(v, torch.Tensor)}
    if c["op"] in ("norm", "quant"):
        t = d["x"]
        if c["op"] == "norm":
            t = d["x"] + d["residual"] if c["residual"] else d["x"]
            ms = torch.einsum("...i,...i->...", t, t) / c["dim"] + EPS
            y = t / ms.sqrt().unsqueeze(-1) * d["weight"].unsqueeze(-2)
        else:
            y = t
        out = {}
        if c["op"] == "quant" or c["e4m3"]:
            out["scale"] = (y.abs().max(dim=-1).values / E4M3_MAX).clamp(min=SCALE_MIN)
            out["q" if c["op"] == "quant" else "y"] = y / out["scale"].unsqueeze(-1)
        else:
            out["y"] = y
        if c["op"] == "norm" and c["residual"]:
            out["sum"] = t
        if c["op"] == "norm" and c["keep"]:
            out["rstd"] = ms.rsqrt()
        return out
    if c["op"] == "norm_bwd":
        # the derivative of y_i = w_i x_i rstd, rstd' = -rstd^3 x / dim
        r, x, dy = d["rstd"].unsqueeze(-1), d["x"], d["dy"]
        along = torch.einsum("...i,...i->...", dy * d["weight"].unsqueeze(-2), x).unsqueeze(-1)
        dx = dy * d["weight"].unsqueeze(-2) * r - along * r ** 3 * x / c["dim"]
        if c["dsum"]:
            dx += d["dsum"]
        return {"dx": dx, "dweight": torch.einsum("...ri,...ri,...r->...i", dy, x, d["rstd"])}
    if c["op"] == "linear":
        x, w = d["x"], d["w"]
        if c["type"] == "e4m3":
            x, w = x * d["x_scale"].unsqueeze(-1), w * d["w_scale"].unsqueeze(-1)
        u = torch.einsum("...mk,...nk->...mn", x, w)
        if c["bias"]:
            u += d["bias"].unsqueeze(-2)
        y = _exact_act(c["act"], u)[0]
        if c["residual"]:
            y = y + d["residual"]
        return {"y": y, "pre": u} if c["keep"] else {"y": y}
    du = d["dy"]
    if c["act"] != "none":
        du = du * _exact_act(c["act"], d["pre"])[1]
    return {"dx": torch.einsum("...mn,...nk->...mk", du, d["w"]),
            "dw": torch.einsum("...mn,...mk->...nk", du, d["x"]), "db": du.sum(dim=-2)}
