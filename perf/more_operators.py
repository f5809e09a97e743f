"""Layer norm and 8-bit activation checkpoints, as cases that can be timed and compared.

    h, s = layernorm(x + s)          a = act(h W1^T + b1)          s' = a W2^T + b2 + s

for one network or for a population of them ("groups", each with weights of its own): the layer norm
with the residual's addition in bf16, fp32 or 8 bits with a scale per row ("norm"), its backward pass
with the gradients of weight and bias ("norm_bwd"), and what a training step keeps for that pass in 8
bits: rows to a checkpoint and back ("checkpoint"), the product that keeps its pre-activations so
("linear"), and its backward pass over them ("linear_bwd"). In a checkpoint 16 adjacent columns share a
power of two, the smallest that is 2^-126 or more and brings them below 127.5, and are rounded to whole
multiples of it.
"""

import math

import torch

own = False  # False: the plain form below; True: the framework's operators

F32, F64, BF16, E4M3 = torch.float32, torch.float64, torch.bfloat16, torch.float8_e4m3fn
E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -126
BLOCK = 16
EPS = 1e-5
SLOPE = 0.2


# ---- cases ------------------------------------------------------------------------------------
def _norm(name, rows, dim, groups=1, type="bf16", residual=True, e4m3=False, keep="none"):
    return _named(name, dict(op="norm", groups=groups, rows=rows, dim=dim, type=type,
                             residual=residual, e4m3=e4m3, keep=keep))


def _norm_bwd(name, rows, dim, groups=1, type="bf16", dsum=True, kept=False):
    return _named(name, dict(op="norm_bwd", groups=groups, rows=rows, dim=dim, type=type, dsum=dsum,
                             kept=kept))


def _checkpoint(name, rows, dim, groups=1, type="bf16", act="none"):
    return _named(name, dict(op="checkpoint", groups=groups, rows=rows, dim=dim, type=type, act=act))


def _linear(name, rows, k, n, groups=1, type="bf16", act="gelu", residual=False, out="bf16"):
    return _named(name, dict(op="linear", groups=groups, rows=rows, k=k, n=n, type=type, act=act,
                             residual=residual, out=out))


def _linear_bwd(name, rows, k, n, groups=1, act="none", kept_x=True):
    return _named(name, dict(op="linear_bwd", groups=groups, rows=rows, k=k, n=n, act=act, kept_x=kept_x))


def _named(name, case):
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one sample through a served network: its norm, in the 8 bits that the next product reads
        _norm("norm_1x4096_e4m3", 1, 4096, e4m3=True),
        # a large batch in training: the sum is kept in 8 bits for the backward pass
        _norm("norm_16384x8192_int8", 16384, 8192, keep="int8"),
        # fp32 rows that are not whole 16-byte units
        _norm("norm_fp32_8193x1001", 8193, 1001, type="fp32", keep="stats"),
        # every cell of a 12x12 grid trains its block: batch 100, hidden width 256
        _norm_bwd("norm_bwd_144x100x256", 100, 256, groups=144),
        # one wide network in training
        _norm_bwd("norm_bwd_8192x4096", 8192, 4096),
        # a large batch whose sum was kept in 8 bits
        _norm_bwd("norm_bwd_int8_16384x2048", 16384, 2048, kept=True),
        # the batch and width of a small ragged network: what it keeps, and back
        _checkpoint("checkpoint_37x500", 37, 500, act="relu"),
        # the pre-activations of a large batch, and the activations worked out from them again
        _checkpoint("checkpoint_16384x4096", 16384, 4096, act="gelu"),
        # the first product of every cell's block
        _linear("linear_144x100x256x512", 100, 256, 512, groups=144),
        # a wide network in training, a large batch
        _linear("linear_8192x4096x8192", 8192, 4096, 8192, act="silu"),
        # sizes that fill no tile, both operands of the weights' gradient from what was kept
        _linear_bwd("linear_bwd_777x500x1001", 777, 500, 1001, act="lrelu"),
        # a wide network in training
        _linear_bwd("linear_bwd_8192x4096x4096", 8192, 4096, 4096, act="gelu"),
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
    op = rng.choice(["norm", "norm", "norm_bwd", "norm_bwd", "checkpoint", "linear", "linear_bwd"])
    groups = rng.choice([1, 1, 1, _log(rng, 2, 144)])
    if op in ("norm", "norm_bwd", "checkpoint"):
        dim, rows, kind = _width(rng, 64, 8192), _rows(rng, 16384), rng.choice(["bf16", "bf16", "fp32"])
        rows = max(1, min(rows, (1 << 26) // (groups * dim)))
        if op == "checkpoint":
            return _checkpoint(None, rows, dim, groups, kind, rng.choice(["none", "relu", "gelu", "silu"]))
        if op == "norm_bwd":
            return _norm_bwd(None, rows, dim, groups, kind, rng.random() < 0.7, rng.random() < 0.4)
        e4m3 = rng.random() < 0.3
        return _norm(None, rows, dim, groups, kind, rng.random() < 0.7, e4m3,
                     rng.choice(["none", "stats", "int8"]))
    k, n, rows = _width(rng, 64, 8192), _width(rng, 16, 8192), _rows(rng, 8192)
    act = rng.choice(["none", "relu", "lrelu", "tanh", "gelu", "silu"])
    rows = max(1, min(rows, (1 << 36) // (groups * k * n)))
    while groups * n * k > 1 << 27:
        groups = groups // 2
    if op == "linear_bwd":
        return _linear_bwd(None, rows, k, n, groups, act, act == "none" or rng.random() < 0.6)
    return _linear(None, rows, k, n, groups, rng.choice(["bf16", "bf16", "e4m3"]), act, rng.random() < 0.3,
                   "fp32" if rng.random() < 0.2 else "bf16")


_TYPES = {"bf16": BF16, "fp32": F32, "e4m3": E4M3}
_BYTES = {"bf16": 2, "fp32": 4, "e4m3": 1}


def _kept_bytes(rows, cols):
    return rows * (cols + -(-cols // BLOCK))


def work(case):
    c = case
    g = c["groups"]
    if c["op"] in ("norm", "norm_bwd", "checkpoint"):
        rows, dim, b = g * c["rows"], c["dim"], _BYTES[c["type"]]
        e, kept = rows * dim, _kept_bytes(rows, dim)
        if c["op"] == "checkpoint":
            return {"bytes": e * b + 2 * kept + e * 2, "flops": 6 * e}
        if c["op"] == "norm":
            moved = e * (b * (1 + 2 * c["residual"]) + (1 if c["e4m3"] else b))
            moved += 8 * g * dim + 4 * rows * (c["e4m3"] + 2 * (c["keep"] != "none"))
            if c["keep"] == "int8":  # written, and read again as the values it stands for
                moved += 2 * kept + 2 * e
            return {"bytes": moved, "flops": 8 * e}
        moved = e * b * (2 + c["dsum"]) + (kept if c["kept"] else e * b) + 8 * rows + 12 * g * dim
        return {"bytes": moved, "flops": 14 * e}
    m, n, k = c["rows"], c["n"], c["k"]
    if c["op"] == "linear":
        b, o = _BYTES[c["type"]], _BYTES[c["out"]]
        moved = g * ((m + n) * k * b + m * n * (o * (1 + c["residual"]) + 2) + 2 * _kept_bytes(m, n))
        moved += g * 4 * (n + ((m + n) if c["type"] == "e4m3" else 0))
        return {"bytes": moved, "flops": 2 * g * m * n * k}
    moved = g * (2 * m * n + (_kept_bytes(m, n) if c["act"] != "none" else 0) + 2 * m * k + 4 * n * k + 4 * n)
    moved += g * (_kept_bytes(m, k) if c["kept_x"] else 2 * m * k)
    return {"bytes": moved, "flops": 4 * g * m * n * k}


# ---- inputs -----------------------------------------------------------------------------------
def _randn(gen, shape, std, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=F32).mul_(std).to(dtype)


def _rows_to_e4m3(x):
    """x in 8 bits with a scale per row, as a served network's weights and inputs are held."""
    scale = (x.float().abs().amax(dim=-1) / E4M3_MAX).clamp_(min=SCALE_MIN)
    return (x.float() / scale[..., None]).to(E4M3), scale


def _blocks(x):
    """[.., columns] as [.., blocks, 16], the last one filled up with zeros."""
    x = torch.nn.functional.pad(x, (0, -x.shape[-1] % BLOCK))
    return x.unflatten(-1, (x.shape[-1] // BLOCK, BLOCK))


def _power(e):
    """2^e in fp32, e in -126..127, from its bits."""
    return ((e + 127) << 23).view(F32)


def _to_blocks(x):
    """(whole multiples, exponents) of x's blocks, in fp32 and int32. (A magnitude's bits order as it does: added
    to them, 2^16 carries into the exponent from 127.5 / 64 of a power of two on.)"""
    v = _blocks(x.float())
    e = (((v.abs().amax(dim=-1).view(torch.int32) + (1 << 16)) >> 23) - 133).clamp(min=-126)
    return torch.round(v * _power(-e)[..., None]), e


def _kept(x):
    """x's checkpoint as a user's program holds it: (whole multiples in int8, exponents + 127 in uint8)."""
    q, e = _to_blocks(x)
    q = q.flatten(-2)[..., :x.shape[-1]]
    return q.to(torch.int8).contiguous(), (e + 127).to(torch.uint8)


def _kept_values(q, scale):
    """The values that a checkpoint stands for, in fp32."""
    unit = _power(scale.to(torch.int32) - 127)
    return (_blocks(q.float()) * unit[..., None]).flatten(-2)[..., :q.shape[-1]]


def _shape(case, *dims):
    return dims if case["groups"] == 1 else (case["groups"],) + dims


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    c, s = case, {"case": case}
    if c["op"] in ("norm", "norm_bwd", "checkpoint"):
        t, rows, dim = _TYPES[c["type"]], c["rows"], c["dim"]
        # (activations have a mean of their own)
        s["x"] = (_randn(gen, _shape(c, rows, dim), 1.0, F32) + 0.5).to(t)
        if c["op"] == "checkpoint":
            return s
        s["weight"] = 1.0 + _randn(gen, _shape(c, dim), 0.1, F32)
        if c["op"] == "norm":
            s["bias"] = _randn(gen, _shape(c, dim), 0.1, F32)
            s["residual"] = _randn(gen, _shape(c, rows, dim), 2.0, t) if c["residual"] else None
            return s
        x = s["x"].float()
        s["mean"] = x.mean(dim=-1)
        s["rstd"] = 1.0 / torch.sqrt((x - s["mean"][..., None]).square().mean(dim=-1) + EPS)
        if c["kept"]:
            s["x"] = _kept(s["x"])
        s["dy"] = _randn(gen, _shape(c, rows, dim), 0.01, t)
        s["dsum"] = _randn(gen, _shape(c, rows, dim), 0.01, t) if c["dsum"] else None
        return s
    m, n, k = c["rows"], c["n"], c["k"]
    x, w = (_randn(gen, _shape(c, m, k), 1.0, BF16), _randn(gen, _shape(c, n, k), k ** -0.5, BF16))
    if c["op"] == "linear":
        s["bias"] = _randn(gen, _shape(c, n), 0.1, F32)
        s["residual"] = (_randn(gen, _shape(c, m, n), 1.0, _TYPES[c["out"]]) if c["residual"] else None)
        if c["type"] == "e4m3":
            (s["x"], s["x_scale"]), (s["w"], s["w_scale"]) = _rows_to_e4m3(x), _rows_to_e4m3(w)
        else:
            s["x"], s["w"], s["x_scale"], s["w_scale"] = x, w, None, None
        return s
    s["x"], s["w"] = _kept(x) if c["kept_x"] else x, w
    s["dy"] = _randn(gen, _shape(c, m, n), 0.01, BF16)
    s["pre"] = _kept(_randn(gen, _shape(c, m, n), 1.0, BF16)) if c["act"] != "none" else None
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


def _through_blocks(x):
    """The values that x's checkpoint stands for: multiples of at most 127 of a power of two, which bf16 holds."""
    q, e = _to_blocks(x)
    return (q * _power(e)[..., None]).flatten(-2)[..., :x.shape[-1]]


def _values(x):
    return _kept_values(*x) if isinstance(x, tuple) else x.float()


def _plain(s):
    c = s["case"]
    if c["op"] == "norm":
        t = _TYPES[c["type"]]
        total = s["x"].float()
        if c["residual"]:
            total = total + s["residual"].float()
        mean = total.mean(dim=-1)
        off = total - mean[..., None]
        rstd = 1.0 / torch.sqrt((off * off).mean(dim=-1) + EPS)
        y = off * rstd[..., None] * s["weight"][..., None, :] + s["bias"][..., None, :]
        out = {}
        if c["e4m3"]:
            out["scale"] = (y.abs().amax(dim=-1) / E4M3_MAX).clamp_(min=SCALE_MIN)
            out["y"] = (y / out["scale"][..., None]).to(E4M3)
        else:
            out["y"] = y.to(t)
        if c["residual"]:
            out["sum"] = total.to(t)
        if c["keep"] != "none":
            out["mean"], out["rstd"] = mean, rstd
        if c["keep"] == "int8":
            out["kept"] = _through_blocks(total.to(t)).to(BF16)
        return out
    if c["op"] == "norm_bwd":
        x, dy, rstd = _values(s["x"]), s["dy"].float(), s["rstd"][..., None]
        x = (x - s["mean"][..., None]) * rstd
        g = dy * s["weight"][..., None, :]
        dx = rstd * (g - g.mean(dim=-1, keepdim=True) - x * (g * x).mean(dim=-1, keepdim=True))
        if c["dsum"]:
            dx = dx + s["dsum"].float()
        return {"dx": dx.to(_TYPES[c["type"]]), "dweight": (dy * x).sum(dim=-2), "dbias": dy.sum(dim=-2)}
    if c["op"] == "checkpoint":
        return {"y": _act(c["act"], _through_blocks(s["x"])).to(BF16)}
    if c["op"] == "linear":
        u = s["x"].float() @ s["w"].float().transpose(-1, -2)
        if c["type"] == "e4m3":
            u = u * s["x_scale"][..., None] * s["w_scale"][..., None, :]
        u = u + s["bias"][..., None, :]
        y = _act(c["act"], u)
        if c["residual"]:
            y = y + s["residual"].float()
        return {"y": y.to(_TYPES[c["out"]]), "pre": _through_blocks(u).to(BF16)}
    du = s["dy"].float()
    if c["act"] != "none":
        du = du * _act_slope(c["act"], _values(s["pre"]))
    return {"dx": (du @ s["w"].float()).to(BF16),
            "dw": (du.transpose(-1, -2) @ _values(s["x"])).to(BF16), "db": du.sum(dim=-2)}


# ---- the framework's operators -------------------------------------------------------------------
def _own(s):
    from paper_1811_12843_gb300 import operators as ops
    c = s["case"]

    def held(x):
        return ops.Checkpoint(*x) if isinstance(x, tuple) else x

    if c["op"] == "norm":
        r = ops.layernorm(s["x"], s["weight"], s["bias"], residual=s["residual"], eps=EPS, e4m3=c["e4m3"],
                          keep={"none": False, "stats": True, "int8": "int8"}[c["keep"]])
        out = {"y": r.y}
        if c["e4m3"]:
            out["scale"] = r.scale
        if c["residual"]:
            out["sum"] = r.sum
        if c["keep"] != "none":
            out["mean"], out["rstd"] = r.mean, r.rstd
        if c["keep"] == "int8":
            out["kept"] = ops.restore_rows(r.kept)
        return out
    if c["op"] == "norm_bwd":
        dx, dweight, dbias = ops.layernorm_backward(s["dy"], held(s["x"]), s["mean"], s["rstd"], s["weight"],
                                                    dsum=s["dsum"])
        return {"dx": dx, "dweight": dweight, "dbias": dbias}
    if c["op"] == "checkpoint":
        return {"y": ops.restore_rows(ops.checkpoint_rows(s["x"]), act=c["act"], slope=SLOPE)}
    if c["op"] == "linear":
        y, pre = ops.linear(s["x"], s["w"], s["bias"], act=c["act"], slope=SLOPE, residual=s["residual"],
                            x_scale=s["x_scale"], w_scale=s["w_scale"], out_dtype=_TYPES[c["out"]],
                            keep="int8")
        return {"y": y, "pre": ops.restore_rows(pre)}
    dx, dw, db = ops.linear_backward(s["dy"], held(s["x"]), s["w"], act=c["act"], slope=SLOPE,
                                     pre=held(s["pre"]))
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


def _power64(e):
    return ((e.to(torch.int64) + 1023) << 52).view(F64)


def _exact_blocks(x):
    """Per 16 columns the unit 2^e, the smallest with e >= -126 that brings them below 127.5, and x's nearest
    multiples of it."""
    cols = x.shape[-1]
    fill = x.new_zeros(x.shape[:-1] + (-cols % BLOCK,))
    v = torch.cat([x, fill], dim=-1)
    v = v.reshape(x.shape[:-1] + (v.shape[-1] // BLOCK, BLOCK))
    top = v.abs().max(dim=-1, keepdim=True).values
    e = torch.floor(torch.log2(top / 127.5)).clamp(min=-126, max=127)
    e = torch.where(top >= 127.5 * _power64(e), e + 1, e)
    unit = _power64(e)
    return (torch.round(v / unit) * unit).reshape(x.shape[:-1] + (-1,))[..., :cols]


def _exact_kept(x):
    if not isinstance(x, tuple):
        return x.to(F64)
    q, scale = x
    unit = _power64(scale.to(torch.int64) - 127)
    column = torch.arange(q.shape[-1], device=q.device) // BLOCK
    return q.to(F64) * unit[..., column]


def exact(case, seed):
    """What run() returns before its one rounding to the output's type (8-bit rows of the norm: the row over
    its scale; checkpoints: the multiples that they hold)."""
    s, c = prepare(case, seed), case
    d = {k: v.to(F64) for k, v in s.items() if isinstance(v, torch.Tensor)}
    if c["op"] == "norm":
        t = d["x"] + d["residual"] if c["residual"] else d["x"]
        mean = torch.einsum("...i->...", t) / c["dim"]
        off = t - mean.unsqueeze(-1)
        var = torch.einsum("...i,...i->...", off, off) / c["dim"] + EPS
        y = off / var.sqrt().unsqueeze(-1) * d["weight"].unsqueeze(-2) + d["bias"].unsqueeze(-2)
        out = {"y": y}
        if c["e4m3"]:
            out["scale"] = (y.abs().max(dim=-1).values / E4M3_MAX).clamp(min=SCALE_MIN)
            out["y"] = y / out["scale"].unsqueeze(-1)
        if c["residual"]:
            out["sum"] = t
        if c["keep"] != "none":
            out["mean"], out["rstd"] = mean, var.rsqrt()
        if c["keep"] == "int8":  # (of the sum as it is written, in the rows' type)
            out["kept"] = _exact_blocks(t.to(F32).to(_TYPES[c["type"]]).to(F64))
        return out
    if c["op"] == "norm_bwd":
        # the derivative of y_i = w_i (x_i - mean) rstd: rstd' = -rstd^3 (x - mean) / dim, mean' = 1 / dim
        r, off, dy = d["rstd"].unsqueeze(-1), _exact_kept(s["x"]) - d["mean"].unsqueeze(-1), d["dy"]
        g = dy * d["weight"].unsqueeze(-2)
        along = torch.einsum("...i,...i->...", g, off).unsqueeze(-1)
        dx = g * r - torch.einsum("...i->...", g).unsqueeze(-1) * r / c["dim"] - along * r ** 3 * off / c["dim"]
        if c["dsum"]:
            dx += d["dsum"]
        return {"dx": dx, "dweight": torch.einsum("...ri,...ri,...r->...i", dy, off, d["rstd"]),
                "dbias": torch.einsum("...ri->...i", dy)}
    if c["op"] == "checkpoint":
        return {"y": _exact_act(c["act"], _exact_blocks(d["x"]))[0]}
    if c["op"] == "linear":
        x, w = d["x"], d["w"]
        if c["type"] == "e4m3":
            x, w = x * d["x_scale"].unsqueeze(-1), w * d["w_scale"].unsqueeze(-1)
        u = torch.einsum("...mk,...nk->...mn", x, w) + d["bias"].unsqueeze(-2)
        y = _exact_act(c["act"], u)[0]
        if c["residual"]:
            y = y + d["residual"]
        return {"y": y, "pre": _exact_blocks(u)}
    du = d["dy"]
    if c["act"] != "none":
        du = du * _exact_act(c["act"], _exact_kept(s["pre"]))[1]
    return {"dx": torch.einsum("...mn,...nk->...mk", du, d["w"]),
            "dw": torch.einsum("...mn,...mk->...nk", du, _exact_kept(s["x"])), "db": du.sum(dim=-2)}
