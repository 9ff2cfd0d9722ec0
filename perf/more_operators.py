"""What a stage of a language model has around its feed-forward products, as a user's program calls it, and in plain torch.

A case names an operator ("op"), its sizes, the type of its tensors and its options:

  join_fwd      s = alpha x + beta gate * drop(post(u)), y = pre(s): a block's result u joins the residual stream x, and the
                next block's input y is made of it (post, pre: norms; gate: none, a vector, or one row for `gate_rows` tokens)
  join_bwd      du, dx, the gradients of both norms' weights and of the gate, from dy and ds
  dropout       y = x keep / (1 - p), with a mask that is a function of (key, step, site, row, column) and is never stored
  rec_fwd       a = sigmoid(f), h_t = a h_(t-1) + (1 - a) v (or + v), y = silu(o) h over sequences, with the last state and, for
                training, the states that the backward pass starts from; one token a sequence is the step of a serving program
  rec_bwd       df, dv, do and the first state's gradient of the same
  logp_fwd      log probabilities of given tokens under rows of logits, their entropy, and the `top` likeliest tokens
  logp_bwd      the gradient of the logits from those of the log probabilities and of the entropies
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6
SITE = 7                 # which dropout of a step this is
KEEP_EVERY = 16          # steps between kept states of the recurrence


def listed():
    def join(name, op, rows, cols, type="bf16", post="rms", pre="rms", gate="vector", gate_rows=0, p=0.0):
        return dict(name=name, op=op, rows=rows, cols=cols, type=type, post=post, pre=pre, gate=gate, gate_rows=gate_rows, p=p)

    def rec(name, op, seqs, steps, cols, type="bf16", ragged=False, coupled=True, gated=True, kept=False):
        return dict(name=name, op=op, seqs=seqs, steps=steps, cols=cols, type=type, ragged=ragged, coupled=coupled, gated=gated, kept=kept)

    def logp(name, op, rows, vocab, type="bf16", top=0, masked=False, entropy=True, scale=1.0):
        return dict(name=name, op=op, rows=rows, vocab=vocab, type=type, top=top, masked=masked, entropy=entropy, scale=scale)
    return [
        # serving: between two blocks of one token, all latency
        join("join fwd, one token", "join_fwd", 1, 4096),
        # training: every term at once, dropout among them
        join("join fwd, 8192 tokens", "join_fwd", 8192, 4096, p=0.1),
        join("join bwd, 8192 tokens", "join_bwd", 8192, 4096, p=0.1),
        # short ragged batch in float, rows off 16 bytes, layer norms, a gate for every sequence of 100 tokens
        join("join bwd, fp32, odd", "join_bwd", 1000, 1283, type="fp32", post="layer", pre="layer", gate="groups", gate_rows=100, p=0.25),
        # activations of a stage's micro-batch
        dict(name="dropout, 16384 tokens", op="dropout", rows=16384, cols=4096, type="bf16", p=0.1),
        dict(name="dropout, fp32, odd", op="dropout", rows=777, cols=1283, type="fp32", p=0.5),
        # serving: one more token of 64 sequences, states updated
        rec("recurrence step, 64 sequences", "rec_fwd", 64, 1, 4096),
        # one long document
        rec("recurrence fwd, 65536 tokens", "rec_fwd", 1, 65536, 2048, kept=True),
        # a packed batch of documents of uneven lengths
        rec("recurrence bwd, ragged", "rec_bwd", 24, 4096, 1536, ragged=True, kept=True),
        # serving: the answer's tokens with their alternatives, part of the vocabulary ruled out
        logp("log probabilities, 16 tokens, top 20", "logp_fwd", 16, 128000, top=20, masked=True, scale=1.25),
        # training: the head's loss over a micro-batch
        logp("log probabilities, 4096 tokens", "logp_fwd", 4096, 50021, entropy=True),
        logp("log probabilities bwd, 8192 tokens", "logp_bwd", 8192, 32000),
    ]


def _spread(rng, lo, hi):
    """A size spread over its logarithm: odd ones as often as multiples of 8 and of 64."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    step = rng.choice((1, 8, 64))
    return min(hi, max(lo, n // step * step or step))


def draw(rng):
    op = rng.choice(("join_fwd", "join_bwd", "dropout", "rec_fwd", "rec_bwd", "logp_fwd", "logp_bwd"))
    while True:
        c = dict(op=op, type=rng.choice(("bf16", "bf16", "fp32")))
        if op in ("join_fwd", "join_bwd"):
            norms = ("rms", "layer")
            c.update(rows=rng.choice((1, 0, 0)) or _spread(rng, 2, 32768), cols=_spread(rng, 32, 16384), post=rng.choice(norms + ("none",)),
                     pre=rng.choice(norms), gate=rng.choice(("none", "vector", "groups")), gate_rows=0, p=rng.choice((0.0, 0.1, 0.3)))
            if c["gate"] == "groups":
                c["gate_rows"] = rng.choice((1, 0)) or _spread(rng, 2, 4096)
        elif op == "dropout":
            c.update(rows=_spread(rng, 1, 65536), cols=_spread(rng, 32, 16384), p=rng.choice((0.05, 0.1, 0.5)))
        elif op in ("rec_fwd", "rec_bwd"):
            steps = 1 if op == "rec_fwd" and rng.random() < 0.3 else _spread(rng, 2, 65536)
            c.update(seqs=_spread(rng, 1, 256), steps=steps, cols=_spread(rng, 32, 8192), ragged=steps > 1 and rng.random() < 0.4,
                     coupled=rng.random() < 0.7, gated=rng.random() < 0.6, kept=op == "rec_bwd" or (steps > 1 and rng.random() < 0.5))
        else:
            c.update(rows=_spread(rng, 1, 16384), vocab=_spread(rng, 100, 256000), top=rng.choice((0, 0, 1, 5, 20)) if op == "logp_fwd" else 0,
                     masked=rng.random() < 0.3, entropy=rng.random() < 0.7, scale=rng.choice((1.0, 1.0, 0.7, 1.5)))
        if work(c)["bytes"] <= 1.0e9:
            return c


def _groups(c):
    return -(-c["rows"] // c["gate_rows"]) if c["gate_rows"] else 1


def _lengths(c):
    """Steps of each sequence: a fixed ragged pattern, an empty sequence and a short one among them."""
    n = c["steps"]
    if not c["ragged"]:
        return [n] * c["seqs"]
    return [0 if i % 11 == 5 else 1 + i % 7 if i % 11 == 8 else max(1, int(n * (1.0 - 0.83 * ((i * 0.618034) % 1.0)))) for i in range(c["seqs"])]


def work(case):
    c, e, op = case, 2 if case["type"] == "bf16" else 4, case["op"]
    if op in ("join_fwd", "join_bwd"):
        n, cols = c["rows"] * c["cols"], c["cols"]
        vectors = 4 * cols * ((c["post"] != "none") * (1 + (c["post"] == "layer")) + 1 + (c["pre"] == "layer"))
        gate = {"none": 0, "vector": 4 * cols, "groups": e * _groups(c) * cols}[c["gate"]]
        if op == "join_fwd":
            return {"bytes": 4 * e * n + vectors + gate, "flops": 15.0 * n}
        return {"bytes": 6 * e * n + 2 * vectors + 2 * gate, "flops": 30.0 * n}
    if op == "dropout":
        return {"bytes": 2 * e * c["rows"] * c["cols"], "flops": 2.0 * c["rows"] * c["cols"]}
    if op in ("rec_fwd", "rec_bwd"):
        rows = sum(_lengths(c))
        n, state = rows * c["cols"], 4 * c["seqs"] * c["cols"]
        kept = 4 * c["cols"] * sum(-(-k // KEEP_EVERY) for k in _lengths(c)) if c["kept"] else 0
        if op == "rec_fwd":
            return {"bytes": e * n * (3 + c["gated"]) + 2 * state + kept, "flops": 10.0 * n}
        return {"bytes": e * n * (5 + 2 * c["gated"]) + 2 * state + kept, "flops": 25.0 * n}
    n = c["rows"] * c["vocab"]
    if op == "logp_fwd":
        return {"bytes": e * n + c["rows"] * (4 + 4 + 8 + 4 * c["entropy"] + 8 * c["top"]), "flops": 6.0 * n}
    return {"bytes": 2 * e * n + c["rows"] * (16 + 8 * c["entropy"]), "flops": 6.0 * n}


# ---- inputs -----------------------------------------------------------------------------------------
def prepare(case, seed):
    c, t, op = case, TYPES[case["type"]], case["op"]
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dev = dict(device="cuda")

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, **dev) * scale

    s = {"case": dict(c)}
    s["rng"] = torch.tensor([0x5EED0000 + int(seed), 1000 + int(seed) % 977], dtype=torch.int64, **dev)      # the key and the step's number
    if op in ("join_fwd", "join_bwd"):
        m, k = c["rows"], c["cols"]
        # the stream has a few channels far above the rest, as networks have them
        loud = torch.where(torch.rand(k, generator=g, **dev) < 0.01, 12.0, 1.0)
        s["u"] = normal(m, k).to(t)
        s["x" if op == "join_fwd" else "s"] = (normal(m, k) * loud).to(t)
        layer = lambda kind: normal(k, scale=0.2) if kind == "layer" else None  # noqa: E731
        s["w_post"] = 1.0 + normal(k, scale=0.2) if c["post"] != "none" else None
        s["b_post"] = layer(c["post"])
        s["w_pre"], s["b_pre"] = 1.0 + normal(k, scale=0.2), layer(c["pre"])
        s["gate"] = {"none": lambda: None, "vector": lambda: 0.5 + normal(k, scale=0.3), "groups": lambda: normal(_groups(c), k).to(t)}[c["gate"]]()
        like = lambda v: None if v is None else torch.empty_like(v)  # noqa: E731
        if op == "join_fwd":
            s["s"], s["y"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
            return s
        s["dy"], s["ds"] = normal(m, k, scale=0.01).to(t), normal(m, k, scale=0.01).to(t)
        stats = torch.zeros(4, m, dtype=torch.float64, **dev)
        for i, (kind, of) in enumerate(((c["post"], "u"), (c["pre"], "s"))):
            v = s[of].double()
            mean = v.mean(1) if kind == "layer" else torch.zeros(m, dtype=torch.float64, **dev)
            stats[2 * i], stats[2 * i + 1] = mean, 1.0 / torch.sqrt(((v - mean[:, None]) ** 2).mean(1) + EPS)
        s["stats"] = stats.float()
        s["du"], s["dx"] = like(s["u"]), like(s["s"])
        for name in ("w_post", "b_post", "w_pre", "b_pre", "gate"):
            s["d" + name] = like(s[name])
        return s
    if op == "dropout":
        s["x"] = normal(c["rows"], c["cols"]).to(t)
        s["y"] = torch.empty_like(s["x"])
        return s
    if op in ("rec_fwd", "rec_bwd"):
        lengths, d = _lengths(c), c["cols"]
        rows = sum(lengths)
        shape = (rows, d) if c["ragged"] else (c["seqs"], c["steps"], d)
        # channels that forget within a few steps beside ones that remember thousands
        s["f"] = (normal(rows, d) + torch.linspace(0.0, 6.0, d, **dev)).to(t).view(shape)
        s["v"] = (normal(rows, d) if c["coupled"] else normal(rows, d, scale=0.05)).to(t).view(shape)
        s["o"] = normal(rows, d).to(t).view(shape) if c["gated"] else None
        s["h0"] = normal(c["seqs"], d, scale=0.3)
        s["offsets"] = torch.tensor([0] + list(np.cumsum(lengths)), dtype=torch.int32, **dev) if c["ragged"] else None
        s["max_len"] = max(lengths)
        s["starts"] = torch.tensor([0] + list(np.cumsum(lengths)), **dev)
        s["long"] = torch.tensor([i for i, n in enumerate(lengths) if n], **dev)                              # sequences that are not empty
        # a kept state's place, and the row it stands in front of
        slots = rows // KEEP_EVERY + c["seqs"]
        first = np.concatenate([[0], np.cumsum(lengths)])
        steps = [np.arange(0, n, KEEP_EVERY) for n in lengths]
        s["kept_rows"] = torch.from_numpy(np.concatenate([first[i] + k for i, k in enumerate(steps)])).to("cuda")
        s["kept_slots"] = torch.from_numpy(np.concatenate([first[i] // KEEP_EVERY + i + k // KEEP_EVERY for i, k in enumerate(steps)])).to("cuda")
        if op == "rec_fwd":
            s["y"], s["h1"] = torch.empty_like(s["v"]), torch.empty_like(s["h0"])
            s["states"] = torch.zeros(slots, d, **dev) if c["kept"] else None
            return s
        s["dy"] = normal(rows, d, scale=0.01).to(t).view(shape)
        s["dh1"] = normal(c["seqs"], d, scale=0.01)
        for name in ("f", "v", "o", "h0"):
            s["d" + name] = torch.empty_like(s[name]) if s[name] is not None else None
        # what the forward pass left: the state in front of every 16th step of a sequence
        f = s["f"].view(rows, d).double()
        a = torch.sigmoid(f)
        h = _scan(a, (torch.sigmoid(-f) if c["coupled"] else 1.0) * s["v"].view(rows, d).double(), s["h0"].double(), s)
        s["states"] = torch.zeros(slots, d, **dev)
        s["states"][s["kept_slots"]] = _before(h.float(), s)[s["kept_rows"]]
        return s
    m, n = c["rows"], c["vocab"]
    z = normal(m, n, scale=2.0)
    z += torch.where(torch.rand(m, n, generator=g, **dev) < 4.0 / n, 8.0, 0.0)                                # a few likely tokens
    if c["masked"]:
        z[:, torch.rand(n, generator=g, **dev) < 0.1] = -math.inf
    noise = -torch.log(-torch.log(torch.rand(m, n, generator=g, **dev).clamp(1e-30, 1.0 - 1e-7)))
    s["targets"] = (z + noise).argmax(1).to(torch.int32)                                                      # drawn from the distribution
    s["logits"] = z.to(t)
    del z, noise
    if op == "logp_fwd":
        f32 = dict(dtype=torch.float32, device="cuda")
        s["logp"], s["lse"] = torch.empty(m, **f32), torch.empty(m, 2, **f32)
        s["entropy"] = torch.empty(m, **f32) if c["entropy"] else None
        s["top"] = torch.empty(m, c["top"], dtype=torch.int32, **dev) if c["top"] else None
        s["top_logp"] = torch.empty(m, c["top"], **f32) if c["top"] else None
        return s
    z = s["logits"].double() * c["scale"]
    top = z.amax(1, keepdim=True)
    lp = z - torch.logsumexp(z, 1, keepdim=True)
    s["lse"] = torch.cat([top / c["scale"], torch.logsumexp(z - top, 1, keepdim=True)], 1).float()           # the largest logit, and the rest of the sum
    s["entropy"] = -(lp.exp() * lp.clamp(min=-1e4)).sum(1).float() if c["entropy"] else None
    del z, lp, top
    s["dlogp"] = normal(m) / m
    s["dentropy"] = normal(m, scale=0.01) / m if c["entropy"] else None
    s["dlogits"] = torch.empty_like(s["logits"])
    return s


# ---- the framework's calls ------------------------------------------------------------------------
def _run_own(s):
    import paper_2110_02781_b200 as F
    c = s["case"]
    op = c["op"]
    if op in ("join_fwd", "join_bwd"):
        norm = {"none": F.NORM_NONE, "rms": F.NORM_RMS, "layer": F.NORM_LAYER}
        how = dict(post=norm[c["post"]], pre=norm[c["pre"]], w_post=s["w_post"], b_post=s["b_post"], w_pre=s["w_pre"], gate=s["gate"],
                   gate_rows=c["gate_rows"], alpha=1.0, beta=0.5, dropout=c["p"], rng=s["rng"] if c["p"] else None, site=SITE)
        if op == "join_fwd":
            F.ftp_join_forward(s["u"], s["x"], s["s"], s["y"], b_pre=s["b_pre"], eps=EPS, **how)
            return {"s": s["s"], "y": s["y"]}
        F.ftp_join_backward(s["u"], s["s"], s["dy"], s["ds"], s["stats"], du=s["du"], dx=s["dx"], dw_post=s["dw_post"], db_post=s["db_post"],
                            dw_pre=s["dw_pre"], db_pre=s["db_pre"], dgate=s["dgate"], **how)
        return {k: s[k] for k in ("du", "dx", "dw_post", "db_post", "dw_pre", "db_pre", "dgate")}
    if op == "dropout":
        F.ftp_dropout(s["x"], s["y"], c["p"], s["rng"], site=SITE)
        return {"y": s["y"]}
    if op in ("rec_fwd", "rec_bwd"):
        how = dict(o=s["o"], act=F.ACT_SILU if c["gated"] else F.ACT_NONE, coupled=c["coupled"], offsets=s["offsets"], max_len=s["max_len"])
        if op == "rec_fwd":
            F.ftp_recurrence_forward(s["f"], s["v"], s["y"], h0=s["h0"], h1=s["h1"], states=s["states"], **how)
            return {"y": s["y"], "h1": s["h1"], "states": s["states"]}
        F.ftp_recurrence_backward(s["f"], s["v"], s["dy"], s["states"], s["df"], s["dv"], do=s["do"], dh1=s["dh1"], dh0=s["dh0"], **how)
        return {"df": s["df"], "dv": s["dv"], "do": s["do"], "dh0": s["dh0"]}
    if op == "logp_fwd":
        F.ftp_logprob_forward(s["logits"], s["targets"], s["logp"], lse=s["lse"], entropy=s["entropy"], top=s["top"], top_logp=s["top_logp"], scale=c["scale"])
        return {k: s[k] for k in ("logp", "lse", "entropy", "top", "top_logp")}
    F.ftp_logprob_backward(s["logits"], s["targets"], s["lse"], s["dlogp"], s["dlogits"], entropy=s["entropy"], dentropy=s["dentropy"], scale=c["scale"])
    return {"dlogits": s["dlogits"]}


# ---- the plain form ---------------------------------------------------------------------------------
def _philox(words, key):
    """Philox 4x32 with ten rounds (Salmon et al., SC 2011) on int64 tensors that hold 32-bit words."""
    def mul(a, b):
        low = a * (b & 0xFFFF)
        high = a * (b >> 16) + (low >> 16)
        return high >> 16, (a * b) & 0xFFFFFFFF
    c0, c1, c2, c3 = words
    k0, k1 = key
    for _ in range(10):
        h0, l0 = mul(c0, 0xD2511F53)
        h1, l1 = mul(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c0, c1, c2, c3


def _keep(rows, cols, p, rng, device):
    """What stays of a rows x cols tensor and the factor it gets.  A call of the generator gives eight neighbouring columns
    16 bits each, so p counts in steps of 2^-16; counter: row and group of eight columns, site, step."""
    cut = int(p * 65536 + 0.5)
    per_row = -(-cols // 8)
    i = torch.arange(rows * per_row, device=device)
    step, key = rng[1], rng[0]
    low = 0xFFFFFFFF
    c2, c3 = (step & low).expand_as(i), ((step >> 32) & low).expand_as(i)
    out = _philox((i & low, (i >> 32) | (SITE << 8), c2, c3), (key & low, (key >> 32) & low))
    u = torch.stack([h for w in out for h in (w & 0xFFFF, w >> 16)], 1).view(rows, per_row * 8)[:, :cols]
    return u >= cut, 65536.0 / (65536 - cut)


def _norm(v, kind, w, b):
    """The normalised rows (without weights), their 1 / deviation, and the weighted result."""
    if kind == "none":
        return v, None, v
    m = v - v.mean(1, keepdim=True) if kind == "layer" else v
    r = 1.0 / torch.sqrt((m * m).mean(1, keepdim=True) + EPS)
    n = m * r
    return n, r, n * w + b if b is not None else n * w


def _norm_bwd(n, r, kind, g):
    """Gradient before a norm from the gradient g of its normalised rows."""
    if kind == "none":
        return g
    d = g - n * (g * n).mean(1, keepdim=True)
    return r * (d - g.mean(1, keepdim=True) if kind == "layer" else d)


def _gate_rows(s, c):
    """The gate's row of every token, in float."""
    if s["gate"] is None:
        return 1.0
    return s["gate"].float().repeat_interleave(c["gate_rows"], 0)[:c["rows"]] if c["gate_rows"] else s["gate"]


def _plain_join(s, c, t):
    m, k = c["rows"], c["cols"]
    u, gate = s["u"].float(), _gate_rows(s, c)
    keep, factor = _keep(m, k, c["p"], s["rng"], u.device) if c["p"] else (None, 1.0)
    n, r, v = _norm(u, c["post"], s["w_post"], s["b_post"])
    drop = lambda a: a if keep is None else torch.where(keep, a * factor, torch.zeros_like(a))  # noqa: E731
    if c["op"] == "join_fwd":
        out = (s["x"].float() + 0.5 * (gate * drop(v))).to(t)                # the stream goes on in the tensors' type
        return {"s": out, "y": _norm(out.float(), c["pre"], s["w_pre"], s["b_pre"])[2].to(t)}
    sv, dy = s["s"].float(), s["dy"].float()
    ns, rs, _ = _norm(sv, c["pre"], s["w_pre"], s["b_pre"])
    d = s["ds"].float() + _norm_bwd(ns, rs, c["pre"], dy * s["w_pre"])
    dv = drop(0.5 * d * gate)
    out = dict(du=_norm_bwd(n, r, c["post"], dv * s["w_post"] if s["w_post"] is not None else dv).to(t), dx=d.to(t), dw_post=None, db_post=None,
               dw_pre=(dy * ns).sum(0), db_pre=dy.sum(0) if s["b_pre"] is not None else None, dgate=None)
    if s["w_post"] is not None:
        out["dw_post"] = (dv * n).sum(0)
    if s["b_post"] is not None:
        out["db_post"] = dv.sum(0)
    if s["gate"] is not None:
        dg = 0.5 * d * drop(v)
        if c["gate_rows"]:
            full = torch.zeros(_groups(c) * c["gate_rows"], k, device=u.device)
            full[:m] = dg
            out["dgate"] = full.view(_groups(c), c["gate_rows"], k).sum(1).to(t)
        else:
            out["dgate"] = dg.sum(0)
    return out


def _scan(a, b, first, s):
    """h_t = a_t h_(t-1) + b_t down the rows, restarted from `first` at every sequence: combined over twice the distance each time."""
    a, h = a.clone(), b.clone()
    at = s["starts"][s["long"]]
    h[at] += a[at] * first[s["long"]]
    a[at] = 0.0
    d = 1
    while d < s["max_len"]:
        h = torch.cat([h[:d], h[d:] + a[d:] * h[:-d]])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return h


def _before(h, s):
    """The state in front of every row."""
    out = torch.cat([h[:1], h[:-1]])
    out[s["starts"][s["long"]]] = s["h0"][s["long"]]
    return out


def _plain_rec(s, c, t):
    d = c["cols"]
    f, v = s["f"].float().reshape(-1, d), s["v"].float().reshape(-1, d)
    a, shape = 1.0 / (1.0 + torch.exp(-f)), s["f"].shape
    other = 1.0 / (1.0 + torch.exp(f))                                        # 1 - a
    h = _scan(a, other * v if c["coupled"] else v, s["h0"], s)
    first, last = s["starts"][s["long"]], s["starts"][s["long"] + 1] - 1
    if c["gated"]:
        o = s["o"].float().reshape(-1, d)
        p = 1.0 / (1.0 + torch.exp(-o))
        gate, dgate = o * p, p * (1.0 + o * (1.0 - p))
    if c["op"] == "rec_fwd":
        h1 = s["h0"].clone()
        h1[s["long"]] = h[last]
        states = None
        if c["kept"]:
            states = torch.zeros_like(s["states"])
            states[s["kept_slots"]] = _before(h, s)[s["kept_rows"]]
        return {"y": (gate * h if c["gated"] else h).to(t).view(shape), "h1": h1, "states": states}
    dy = s["dy"].float().reshape(-1, d)
    before = _before(h, s)
    e = dy * gate if c["gated"] else dy.clone()
    e[last] += s["dh1"][s["long"]]
    after = torch.cat([a[1:], torch.zeros_like(a[:1])])                       # the decay of the step behind
    after[last] = 0.0
    after, delta, k = after.flip(0), e.flip(0), 1
    while k < s["max_len"]:
        delta = torch.cat([delta[:k], delta[k:] + after[k:] * delta[:-k]])
        after = torch.cat([after[:k], after[k:] * after[:-k]])
        k *= 2
    delta = delta.flip(0)
    dh0 = s["dh1"].clone()
    dh0[s["long"]] = a[first] * delta[first]
    da = delta * (before - v) if c["coupled"] else delta * before
    return {"df": (da * a * other).to(t).view(shape), "dv": (delta * other if c["coupled"] else delta).to(t).view(shape),
            "do": (dy * h * dgate).to(t).view(shape) if c["gated"] else None, "dh0": dh0}


def _plain_logp(s, c, t):
    z = s["logits"].float() * c["scale"]
    at = s["targets"].long()[:, None]
    if c["op"] == "logp_fwd":
        top = z.amax(1, keepdim=True)
        e = torch.exp(z - top)
        total = e.sum(1, keepdim=True)
        lse = top + torch.log(total)
        out = dict(logp=(z.gather(1, at) - lse)[:, 0], lse=torch.cat([s["logits"].float().amax(1, keepdim=True), torch.log(total)], 1), entropy=None, top=None, top_logp=None)
        if c["entropy"]:
            low = torch.where(e > 0, z - lse, torch.zeros_like(z))
            out["entropy"] = -(e / total * low).sum(1)
        if c["top"]:
            value, index = torch.sort(z, dim=1, descending=True, stable=True)  # of equal ones the lowest token first
            out["top"], out["top_logp"] = index[:, :c["top"]].to(torch.int32), value[:, :c["top"]] - lse
        return out
    lp = (s["logits"].float() - s["lse"][:, :1]) * c["scale"] - s["lse"][:, 1:]
    p = torch.exp(lp)
    d = -p * s["dlogp"][:, None]
    d.scatter_add_(1, at, s["dlogp"][:, None])
    if c["entropy"]:
        d = d - s["dentropy"][:, None] * p * torch.where(p > 0, lp + s["entropy"][:, None], torch.zeros_like(p))
    return {"dlogits": (d * c["scale"]).to(t)}


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    t, op = TYPES[c["type"]], c["op"]
    if op in ("join_fwd", "join_bwd"):
        return _plain_join(state, c, t)
    if op == "dropout":
        x = state["x"].float()
        keep, factor = _keep(c["rows"], c["cols"], c["p"], state["rng"], x.device)
        return {"y": torch.where(keep, x * factor, torch.zeros_like(x)).to(t)}
    if op in ("rec_fwd", "rec_bwd"):
        return _plain_rec(state, c, t)
    return _plain_logp(state, c, t)


# ---- the definition in 64 bits -----------------------------------------------------------------------
def _mask64(rows, cols, p, rng):
    """The same generator on numpy's 64-bit words: the factor of every element."""
    per_row = (cols + 7) // 8
    key, step = (int(v) & 0xFFFFFFFFFFFFFFFF for v in rng.tolist())
    n = np.arange(rows * per_row, dtype=np.uint64)
    u32, low = np.uint64(32), np.uint64(0xFFFFFFFF)
    a, b = n & low, (n >> u32) | np.uint64(SITE * 256)
    x, y = np.full_like(n, step & 0xFFFFFFFF), np.full_like(n, step >> 32)
    ka, kb = key & 0xFFFFFFFF, key >> 32
    for _ in range(10):
        pa, px = a * np.uint64(0xD2511F53), x * np.uint64(0xCD9E8D57)
        a, b, x, y = (px >> u32) ^ b ^ np.uint64(ka), px & low, (pa >> u32) ^ y ^ np.uint64(kb), pa & low
        ka, kb = (ka + 0x9E3779B9) % 2 ** 32, (kb + 0xBB67AE85) % 2 ** 32
    bits = np.empty((rows * per_row, 8), np.int32)
    for i, w in enumerate((a, b, x, y)):
        bits[:, 2 * i], bits[:, 2 * i + 1] = w & np.uint64(65535), w >> np.uint64(16)
    cut = int(math.floor(p * 65536 + 0.5))
    kept = torch.from_numpy((bits >= cut).reshape(rows, -1)[:, :cols].copy()).cuda()
    return kept.double() * (65536.0 / (65536.0 - cut))


def _exact_join(s, c, t):
    d = {k: v.double() for k, v in s.items() if torch.is_tensor(v) and k != "rng"}
    m, k = c["rows"], c["cols"]
    mask = _mask64(m, k, c["p"], s["rng"]) if c["p"] else torch.ones(m, k, dtype=torch.float64, device="cuda")
    of_row = torch.arange(m, device="cuda") // max(1, c["gate_rows"])
    gate = torch.ones(k, dtype=torch.float64, device="cuda") if s["gate"] is None else d["gate"][of_row] if c["gate_rows"] else d["gate"]

    def unit(v, kind):
        if kind == "none":
            return v, None
        mu = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros(v.shape[0], 1, dtype=v.dtype, device=v.device)
        sigma = (((v - mu) ** 2).mean(1, keepdim=True) + EPS).sqrt()
        return (v - mu) / sigma, sigma

    def affine(n, w, b):
        n = n * d[w] if w in d else n
        return n + d[b] if b in d else n

    def back(n, sigma, kind, g):
        if kind == "none":
            return g
        inner = torch.sum(g * n, 1, keepdim=True) / k
        mean = torch.sum(g, 1, keepdim=True) / k if kind == "layer" else 0.0
        return (g - mean - n * inner) / sigma

    un, us = unit(d["u"], c["post"])
    branch = mask * affine(un, "w_post", "b_post")
    if c["op"] == "join_fwd":
        out = d["x"] + gate * branch / 2
        return {"s": out, "y": affine(unit(out.to(t).double(), c["pre"])[0], "w_pre", "b_pre")}
    sn, ss = unit(d["s"], c["pre"])
    total = d["ds"] + back(sn, ss, c["pre"], d["dy"] * d["w_pre"])
    dv = total * gate * mask / 2
    res = {"du": back(un, us, c["post"], dv * d["w_post"] if "w_post" in d else dv), "dx": total, "dw_post": None, "db_post": None,
           "dw_pre": torch.sum(d["dy"] * sn, 0), "db_pre": torch.sum(d["dy"], 0) if "b_pre" in d else None, "dgate": None}
    if "w_post" in d:
        res["dw_post"] = torch.sum(dv * un, 0)
    if "b_post" in d:
        res["db_post"] = torch.sum(dv, 0)
    if "gate" in d:
        each = total * branch / 2
        res["dgate"] = torch.zeros_like(d["gate"]).index_add_(0, of_row, each) if c["gate_rows"] else torch.sum(each, 0)
    return res


def _exact_rec(s, c):
    """Step by step in time, all sequences at once."""
    d = c["cols"]
    lengths = _lengths(c)
    order = sorted(range(c["seqs"]), key=lambda i: -lengths[i])
    starts = s["starts"][:-1][torch.tensor(order, device="cuda")]
    active = [0] * (max(lengths) + 1)
    for n in lengths:
        active[n] += 1
    count, alive = len(lengths), []
    for t in range(max(lengths)):
        count -= active[t]
        alive.append(count)
    flat = {k: s[k].double().reshape(-1, d) for k in ("f", "v", "o", "dy") if s.get(k) is not None}
    a = torch.sigmoid(flat["f"])
    b = torch.sigmoid(-flat["f"])
    drive = b * flat["v"] if c["coupled"] else flat["v"]
    perm = torch.tensor(order, device="cuda")
    h = s["h0"].double()[perm].clone()
    hs, before = torch.empty_like(a), torch.empty_like(a)
    for t, n in enumerate(alive):
        rows = starts[:n] + t
        before[rows] = h[:n]
        h[:n] = a[rows] * h[:n] + drive[rows]
        hs[rows] = h[:n]
    back = torch.empty_like(perm)
    back[perm] = torch.arange(len(order), device="cuda")
    shape = s["f"].shape
    if c["gated"]:
        sig = torch.sigmoid(flat["o"])
        gate, slope = flat["o"] * sig, sig + flat["o"] * sig * torch.sigmoid(-flat["o"])
    if c["op"] == "rec_fwd":
        kept = None
        if c["kept"]:
            kept = torch.zeros(s["states"].shape, dtype=torch.float64, device="cuda")
            kept[s["kept_slots"]] = before[s["kept_rows"]]
        return {"y": (gate * hs if c["gated"] else hs).view(shape), "h1": h[back], "states": kept}
    q = s["dh1"].double()[perm].clone()
    into = flat["dy"] * gate if c["gated"] else flat["dy"]
    delta = torch.empty_like(a)
    for t in range(len(alive) - 1, -1, -1):
        n = alive[t]
        rows = starts[:n] + t
        g = into[rows] + q[:n]
        delta[rows] = g
        q[:n] = a[rows] * g
    da = delta * (before - flat["v"]) if c["coupled"] else delta * before
    return {"df": (da * a * b).view(shape), "dv": (delta * b if c["coupled"] else delta).view(shape),
            "do": (flat["dy"] * hs * slope).view(shape) if c["gated"] else None, "dh0": q[back]}


def _exact_logp(s, c):
    z = torch.mul(s["logits"].double(), c["scale"])
    rows = torch.arange(c["rows"], device="cuda")
    lse = torch.logsumexp(z, 1)
    lp = z - lse.unsqueeze(1)
    p = torch.exp(lp)
    plogp = torch.where(torch.isinf(lp), torch.zeros_like(p), p * lp)
    if c["op"] == "logp_fwd":
        res = {"logp": lp[rows, s["targets"].long()], "lse": torch.stack([s["logits"].double().max(1).values, lse - z.max(1).values], 1), "entropy": -plogp.sum(1) if c["entropy"] else None, "top": None, "top_logp": None}
        if c["top"]:
            index = torch.sort(-s["logits"].double(), dim=1, stable=True)[1][:, :c["top"]]
            res["top"], res["top_logp"] = index.to(torch.int32), torch.gather(lp, 1, index)
        return res
    g = -p * s["dlogp"].double()[:, None]
    g[rows, s["targets"].long()] += s["dlogp"].double()
    if c["entropy"]:
        g -= s["dentropy"].double()[:, None] * (plogp - p * plogp.sum(1, keepdim=True))
    return {"dlogits": g * c["scale"]}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("join_fwd", "join_bwd"):
        return _exact_join(s, case, TYPES[case["type"]])
    if op == "dropout":
        return {"y": s["x"].double() * _mask64(case["rows"], case["cols"], case["p"], s["rng"])}
    if op in ("rec_fwd", "rec_bwd"):
        return _exact_rec(s, case)
    return _exact_logp(s, case)
