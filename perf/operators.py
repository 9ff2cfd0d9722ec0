"""The feed-forward operators as a user's program calls them, and the same operators in plain torch.

A case names an operator ("op"), its sizes (rows = tokens, cin, cout), the type of its tensors and its options:

  linear_fwd   y = act(x w + b) + r, with the values before the activation kept for the backward pass ("stash") or not
  linear_bwd   dx, dw, db of the same from dy and the kept values
  gated_fwd    h = act(x wg) * (x wu), both projections' results kept or not
  gated_bwd    dx, dwg, dwu of the same from dh and the kept values
  checkpoint   an activation packed to 8 bits (one power-of-two scale per 32 columns) and unpacked again
  block        a training step of a gated feed-forward block, y = (act(x wg) * (x wu)) wd + x, that keeps x, h and both
               projections' results in 8 bits only and takes its gradients from them
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BLOCK = 32          # columns that share a scale in 8 bits


def listed():
    def case(name, op, rows, cin, cout, type="bf16", act="none", bias=False, residual=False, stash=False):
        return dict(name=name, op=op, rows=rows, cin=cin, cout=cout, type=type, act=act, bias=bias, residual=residual, stash=stash)
    return [
        # serving: the output projection of one token, bound by reading the weights and by latency
        case("linear fwd, one token", "linear_fwd", 1, 4096, 4096, act="gelu", bias=True, residual=True),
        # training, or a batch of prompts: every term of the epilogue, and the kept values
        case("linear fwd, 8192 tokens", "linear_fwd", 8192, 4096, 4096, act="gelu", bias=True, residual=True, stash=True),
        # float tensors with odd widths: rows that do not start on 16 bytes
        case("linear fwd, fp32, odd", "linear_fwd", 1000, 1283, 517, type="fp32", act="silu", bias=True, residual=True),
        case("linear bwd, 8192 tokens", "linear_bwd", 8192, 4096, 4096, act="gelu", bias=True),
        # the width of the last 1x1 convolution and classifier of the 224 x 224 network, in float
        case("linear bwd, fp32", "linear_bwd", 2048, 1280, 1000, type="fp32", act="relu6", bias=True),
        case("gated fwd, one token", "gated_fwd", 1, 4096, 12288, act="silu"),
        case("gated fwd, 8192 tokens", "gated_fwd", 8192, 4096, 12288, act="silu", stash=True),
        case("gated bwd, 8192 tokens", "gated_bwd", 8192, 4096, 12288, act="silu"),
        # a short ragged batch in float
        case("gated bwd, fp32, ragged", "gated_bwd", 777, 1000, 2730, type="fp32", act="gelu"),
        # a stage's input kept for its backward pass
        case("checkpoint, 16384 tokens", "checkpoint", 16384, 4096, 0),
        case("checkpoint, fp32, ragged", "checkpoint", 333, 1283, 0, type="fp32"),
        # a stage of the pipeline that holds its micro-batch in 8 bits between the passes
        case("block, 4096 tokens", "block", 4096, 2048, 8192, act="silu"),
    ]


def _spread(rng, lo, hi):
    """A size spread over its logarithm: odd ones as often as multiples of 8 and of 64."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    step = rng.choice((1, 8, 64))
    return min(hi, max(lo, n // step * step or step))


def draw(rng):
    op = rng.choice(("linear_fwd", "linear_fwd", "linear_bwd", "gated_fwd", "gated_fwd", "gated_bwd", "checkpoint", "block"))
    while True:
        rows = rng.choice((1, 1, 0)) or _spread(rng, 2, 16384)
        c = dict(op=op, rows=rows if op in ("linear_fwd", "gated_fwd") else _spread(rng, 2, 16384), cin=_spread(rng, 32, 8192), cout=_spread(rng, 32, 16384),
                 type=rng.choice(("bf16", "bf16", "fp32")), act=rng.choice(("relu", "relu6", "gelu", "silu", "none")), bias=False, residual=False, stash=False)
        if op == "checkpoint":
            c["cout"], c["act"] = 0, "none"
        if op == "block":
            c["type"] = "bf16"      # float results taken from 8 bits turn on the last bit of every value next to a rounding border
        if op in ("linear_fwd", "linear_bwd"):
            c["bias"] = rng.random() < 0.7
        if op == "linear_fwd":
            c["residual"] = rng.random() < 0.5
        if op in ("linear_fwd", "gated_fwd"):
            c["stash"] = c["rows"] > 1 and c["act"] != "none" and rng.random() < 0.5
        w = work(c)
        if w["flops"] <= 1.5e12 and w["bytes"] <= 1.5e9:
            return c


def work(case):
    m, k, n, e = case["rows"], case["cin"], case["cout"], 2 if case["type"] == "bf16" else 4
    eight = lambda rows, cols: rows * (cols + -(-cols // BLOCK))  # noqa: E731
    op = case["op"]
    if op == "linear_fwd":
        return {"bytes": e * (m * k + k * n + m * n * (1 + case["residual"] + case["stash"])) + 4 * n * case["bias"], "flops": 2.0 * m * k * n}
    if op == "linear_bwd":
        kept = case["act"] != "none"
        return {"bytes": e * (2 * m * k + 2 * k * n + m * n * (1 + kept)) + 4 * n * case["bias"], "flops": 4.0 * m * k * n}
    if op == "gated_fwd":
        return {"bytes": e * (m * k + 2 * k * n + m * n * (1 + 2 * case["stash"])), "flops": 4.0 * m * k * n}
    if op == "gated_bwd":
        return {"bytes": e * (2 * m * k + 4 * k * n + 3 * m * n), "flops": 8.0 * m * k * n}
    if op == "checkpoint":
        return {"bytes": e * 2 * m * k + 2 * eight(m, k), "flops": 0.0}
    # block: x, dy in and y, dx out; three weights read in each direction and their gradients; the 8-bit images written and read
    return {"bytes": e * (4 * m * k + 9 * k * n) + 2 * (eight(m, k) + 3 * eight(m, n)), "flops": 18.0 * m * k * n}


def prepare(case, seed):
    m, k, n, t = case["rows"], case["cin"], case["cout"], TYPES[case["type"]]
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dev = dict(device="cuda")

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, **dev) * scale

    # activations with a few channels far above the rest, as networks have them
    x = normal(m, k) * torch.where(torch.rand(k, generator=g, **dev) < 0.01, 12.0, 1.0)
    s = {"case": dict(case), "x": x.to(t)}
    op = case["op"]
    if op == "checkpoint":
        s["out"] = torch.empty_like(s["x"])
        return s
    w = lambda a, b: normal(a, b, scale=a ** -0.5).to(t)  # noqa: E731
    f32 = torch.float32
    if op in ("linear_fwd", "linear_bwd"):
        s["w"] = w(k, n)
        s["bias"] = normal(n, scale=0.1) if case["bias"] else None
    else:
        s["wg"], s["wu"] = w(k, n), w(k, n)
    if op == "linear_fwd":
        s["residual"] = normal(m, n).to(t) if case["residual"] else None
        s["y"] = torch.empty(m, n, dtype=t, **dev)
        s["pre"] = torch.empty(m, n, dtype=t, **dev) if case["stash"] else None
    elif op == "linear_bwd":
        s["pre"] = normal(m, n, scale=1.5).to(t) if case["act"] != "none" else None
        s["dy"] = normal(m, n, scale=0.01).to(t)
        s["dx"], s["dw"] = torch.empty(m, k, dtype=t, **dev), torch.empty(k, n, dtype=t, **dev)
        s["dbias"] = torch.empty(n, dtype=f32, **dev) if case["bias"] else None
    elif op == "gated_fwd":
        s["h"] = torch.empty(m, n, dtype=t, **dev)
        s["pre"] = torch.empty(2, m, n, dtype=t, **dev) if case["stash"] else None
    elif op == "gated_bwd":
        s["pre"] = normal(2, m, n, scale=1.5).to(t)
        s["dh"] = normal(m, n, scale=0.01).to(t)
        s["dx"] = torch.empty(m, k, dtype=t, **dev)
        s["dwg"], s["dwu"] = torch.empty(k, n, dtype=t, **dev), torch.empty(k, n, dtype=t, **dev)
    else:
        s["wd"] = w(n, k)
        s["dy"] = normal(m, k, scale=0.01).to(t)
        for name, shape in (("h", (m, n)), ("dh", (m, n)), ("y", (m, k)), ("dx", (m, k)), ("dwg", (k, n)), ("dwu", (k, n)), ("dwd", (n, k))):
            s[name] = torch.empty(*shape, dtype=t, **dev)
    return s


# ---- the framework's calls ------------------------------------------------------------------------
def _run_own(s):
    import paper_2110_02781_b200 as F
    c = s["case"]
    op, act = c["op"], getattr(F, "ACT_" + c["act"].upper())
    if op == "linear_fwd":
        F.ftp_linear_forward(s["x"], s["w"], s["y"], bias=s["bias"], residual=s["residual"], act=act, stash=s["pre"])
        return {"y": s["y"], "pre": s["pre"]}
    if op == "linear_bwd":
        F.ftp_linear_backward(s["x"], s["w"], s["dy"], dx=s["dx"], dw=s["dw"], dbias=s["dbias"], act=act, stash=s["pre"])
        return {"dx": s["dx"], "dw": s["dw"], "dbias": s["dbias"]}
    if op == "gated_fwd":
        F.ftp_gated_forward(s["x"], s["wg"], s["wu"], s["h"], act=act, stash=s["pre"])
        return {"h": s["h"], "pre": s["pre"]}
    if op == "gated_bwd":
        F.ftp_gated_backward(s["x"], s["wg"], s["wu"], s["dh"], dx=s["dx"], dw_gate=s["dwg"], dw_up=s["dwu"], act=act, stash=s["pre"])
        return {"dx": s["dx"], "dwg": s["dwg"], "dwu": s["dwu"]}
    image = lambda rows, cols, parts=1: torch.empty(F.ftp_checkpoint_bytes(rows, cols, parts), dtype=torch.uint8, device="cuda")  # noqa: E731
    m, k, n = c["rows"], c["cin"], c["cout"]
    x8 = image(m, k)
    F.ftp_checkpoint_pack(s["x"], x8)
    if op == "checkpoint":
        F.ftp_checkpoint_unpack(x8, s["out"])
        return {"out": s["out"]}
    pre8, h8 = image(m, n, 2), image(m, n)
    F.ftp_gated_forward(s["x"], s["wg"], s["wu"], s["h"], act=act, stash=pre8)
    F.ftp_checkpoint_pack(s["h"], h8)
    F.ftp_linear_forward(s["h"], s["wd"], s["y"], residual=s["x"])
    F.ftp_linear_backward(h8, s["wd"], s["dy"], dx=s["dh"], dw=s["dwd"])
    F.ftp_gated_backward(x8, s["wg"], s["wu"], s["dh"], dx=s["dx"], dw_gate=s["dwg"], dw_up=s["dwu"], act=act, stash=pre8, dx_addend=s["dy"])
    return {"y": s["y"], "dx": s["dx"], "dwg": s["dwg"], "dwu": s["dwu"], "dwd": s["dwd"]}


# ---- the plain form ---------------------------------------------------------------------------------
def _act(z, act):
    """The activation and its derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        on = (z > 0).to(z.dtype)
        return z * on, on
    if act == "relu6":
        return z.clamp(0.0, 6.0), ((z > 0) & (z < 6)).to(z.dtype)
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return z * p, p * (1.0 + z * (1.0 - p))
    p = 0.5 * (1.0 + torch.erf(z * 0.7071067811865476))
    return z * p, p + z * torch.exp(-0.5 * z * z) * 0.3989422804014327


def _through_8_bits(x):
    """x as its 8-bit image gives it back: whole multiples of a power of two per BLOCK columns, in -127..127."""
    rows, cols = x.shape
    xb = torch.zeros(rows, -(-cols // BLOCK) * BLOCK, dtype=torch.float32, device=x.device)
    xb[:, :cols] = x
    xb = xb.view(rows, -1, BLOCK)
    top = xb.abs().amax(2, keepdim=True)
    _, e = torch.frexp(top)                                   # top in [2^(e-1), 2^e)
    scale = ((e.clamp(min=-119) - 7 + 127) << 23).view(torch.float32)
    q = torch.round(xb / scale).clamp(-127, 127)
    return (q * scale).view(rows, -1)[:, :cols]


def _run_plain(s):
    c = s["case"]
    op, act, t = c["op"], c["act"], TYPES[c["type"]]
    x = s["x"].float()
    if op == "linear_fwd":
        z = x @ s["w"].float()
        if s["bias"] is not None:
            z = z + s["bias"]
        y = _act(z, act)[0]
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(t), "pre": z.to(t) if s["pre"] is not None else None}
    if op == "linear_bwd":
        dz = s["dy"].float()
        if s["pre"] is not None:
            dz = dz * _act(s["pre"].float(), act)[1]
        return {"dx": (dz @ s["w"].float().T).to(t), "dw": (x.T @ dz).to(t), "dbias": dz.sum(0) if s["dbias"] is not None else None}
    if op == "checkpoint":
        return {"out": _through_8_bits(x).to(t)}
    wg, wu = s["wg"].float(), s["wu"].float()
    if op == "gated_fwd":
        g, u = x @ wg, x @ wu
        return {"h": (_act(g, act)[0] * u).to(t), "pre": torch.stack((g, u)).to(t) if s["pre"] is not None else None}
    if op == "gated_bwd":
        g, u, dh = s["pre"][0].float(), s["pre"][1].float(), s["dh"].float()
        a, da = _act(g, act)
        dg, du = dh * u * da, dh * a
        return {"dx": (dg @ wg.T + du @ wu.T).to(t), "dwg": (x.T @ dg).to(t), "dwu": (x.T @ du).to(t)}
    wd, dy = s["wd"].float(), s["dy"].float()
    g, u = x @ wg, x @ wu
    h = (_act(g, act)[0] * u).to(t).float()                     # h goes from one operator to the next in the tensors' type
    y = (h @ wd + x).to(t)
    x8, h8, g8, u8 = _through_8_bits(x), _through_8_bits(h), _through_8_bits(g), _through_8_bits(u)
    dh = (dy @ wd.T).to(t).float()                              # and so does its gradient
    a, da = _act(g8, act)
    dg, du = dh * u8 * da, dh * a
    return {"y": y, "dx": (dg @ wg.T + du @ wu.T + dy).to(t), "dwg": (x8.T @ dg).to(t), "dwu": (x8.T @ du).to(t), "dwd": (h8.T @ dy).to(t)}


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


# ---- the definition in 64 bits -----------------------------------------------------------------------
def _phi64(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def _f64(z, act):
    return {"none": lambda: z, "relu": lambda: torch.relu(z), "relu6": lambda: torch.minimum(torch.relu(z), torch.full_like(z, 6.0)),
            "silu": lambda: z * torch.sigmoid(z), "gelu": lambda: z * _phi64(z)}[act]()


def _df64(z, act):
    one, zero = torch.ones_like(z), torch.zeros_like(z)
    if act == "none":
        return one
    if act == "relu":
        return torch.where(z > 0, one, zero)
    if act == "relu6":
        return torch.where((z > 0) & (z < 6), one, zero)
    if act == "silu":
        return torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
    return _phi64(z) + z * torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)


def _eight64(x):
    out = x.clone()
    cols = x.shape[1]
    whole = cols // BLOCK * BLOCK
    for a, b, width in ((0, whole, BLOCK), (whole, cols, cols - whole)):
        if a == b:
            continue
        v = x[:, a:b].reshape(x.shape[0], -1, width)
        top = v.abs().max(dim=2, keepdim=True).values
        low = torch.floor(torch.log2(top.clamp(min=2.0 ** -120)))
        low = torch.where(torch.exp2(low) > top, low - 1, low)  # the whole power of two at or below the largest value
        low = torch.where(torch.exp2(low + 1) <= top, low + 1, low).clamp(min=-120)
        step = torch.exp2(torch.round(low) - 6)
        out[:, a:b] = (torch.clamp(torch.round(v / step), -127, 127) * step).reshape(x.shape[0], -1)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    d = {key: v.double() for key, v in s.items() if torch.is_tensor(v)}
    op, act, t = case["op"], case["act"], TYPES[case["type"]]
    x = d["x"]
    if op == "linear_fwd":
        z = torch.addmm(d["bias"], x, d["w"]) if case["bias"] else torch.mm(x, d["w"])
        y = _f64(z, act)
        return {"y": y + d["residual"] if case["residual"] else y, "pre": z if case["stash"] else None}
    if op == "linear_bwd":
        dz = d["dy"] * _df64(d["pre"], act) if act != "none" else d["dy"]
        return {"dx": torch.mm(dz, d["w"].T), "dw": torch.mm(x.T, dz), "dbias": torch.sum(dz, 0) if case["bias"] else None}
    if op == "checkpoint":
        return {"out": _eight64(x)}
    if op == "gated_fwd":
        g, u = torch.mm(x, d["wg"]), torch.mm(x, d["wu"])
        return {"h": _f64(g, act) * u, "pre": torch.stack([g, u]) if case["stash"] else None}
    if op == "gated_bwd":
        g, u, dh = d["pre"][0], d["pre"][1], d["dh"]
        dg, du = dh * u * _df64(g, act), dh * _f64(g, act)
        return {"dx": torch.addmm(torch.mm(dg, d["wg"].T), du, d["wu"].T), "dwg": torch.mm(x.T, dg), "dwu": torch.mm(x.T, du)}
    as_type = lambda v: v.to(t).double()  # noqa: E731   what one operator hands to the next is in the tensors' type
    g, u = torch.mm(x, d["wg"]), torch.mm(x, d["wu"])
    h = as_type(_f64(g, act) * u)
    dh = as_type(torch.mm(d["dy"], d["wd"].T))
    g8, u8, x8 = _eight64(g), _eight64(u), _eight64(x)
    dg, du = dh * u8 * _df64(g8, act), dh * _f64(g8, act)
    return {"y": torch.mm(h, d["wd"]) + x, "dx": torch.mm(dg, d["wg"].T) + torch.mm(du, d["wu"].T) + d["dy"],
            "dwg": torch.mm(x8.T, dg), "dwu": torch.mm(x8.T, du), "dwd": torch.mm(_eight64(h).T, d["dy"])}
