"""Operators around the feed-forward products on the GPU: block joins, dropout, gated recurrence, log probabilities of tokens."""
import math
import subprocess
import sys
import threading
import zlib
from pathlib import Path

import pytest
import torch

import token_helpers as H
from ffn_helpers import ACTS, HALF, Guarded, act, assert_within, dact

F = pytest.importorskip("paper_2110_02781_b200")
pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def rnd(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, dtype=torch.float64) * scale


def on_gpu(t, dt, gap=0, off=0):
    """A rows x cols tensor of type dt on the GPU with a gap behind every row, and its values in float64."""
    g = Guarded(t.shape[0], t.shape[1], dt, gap, off, fill=t.to(dt))
    return g, t.to(dt).double()


def vec(t):
    return (None, None) if t is None else (t.float().cuda(), t.float().double())


def rng_of(key, step):
    return torch.tensor([key, step], dtype=torch.int64, device="cuda")


def close(got, pair, dt, what):
    ref, bound = pair
    assert_within(got, ref, bound + HALF[dt] * ref.abs() + 1e-37, what)


# ---- dropout ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,cols,gap,off", [(1, 1, 0, 0), (1, 8, 0, 0), (3, 7, 0, 0), (2, 31, 3, 1), (5, 256, 8, 0), (7, 257, 0, 0), (129, 1283, 5, 1), (300, 96, 0, 8), (9, 5000, 0, 0)])
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("p", [0.1, 0.5])
def test_dropout(rows, cols, gap, off, dt, p):
    g = gen(rows, cols, p)
    x, x64 = on_gpu(rnd(g, rows, cols), dt, gap, off)
    y = Guarded(rows, cols, dt, gap, 0)
    F.ftp_dropout(x.t, y.t, p, rng_of(-(5 << 40) + 7, 3), site=9, row0=1000)
    keep, f = H.keep_mask(rows, cols, p, -(5 << 40) + 7, 3, 9, 1000)
    close(y.t, (torch.where(keep, x64 * f, torch.zeros_like(x64)), 2 * H.U * (x64 * f).abs()), dt, "y")
    assert y.untouched() and bool(((y.t != 0).cpu() == keep).all())


def test_dropout_rates_parts_and_what_is_dropped():
    x = torch.randn(64, 1000, device="cuda")
    words = rng_of(1, 2)
    y = torch.empty_like(x)
    F.ftp_dropout(x, y, 0.0, None)
    assert torch.equal(x, y)
    F.ftp_dropout(x, y, 1.0, words)
    assert not y.any()
    F.ftp_dropout(x, y, 0.3, words, site=4)
    parts = torch.empty_like(x)
    for a, b in ((0, 10), (10, 11), (11, 64)):                          # micro-batches
        F.ftp_dropout(x[a:b], parts[a:b], 0.3, words, site=4, row0=a)
    assert torch.equal(y, parts)
    F.ftp_dropout(parts.copy_(x), parts, 0.3, words, site=4)            # in place
    assert torch.equal(y, parts)
    for other in (dict(site=5), dict(row0=64)):
        F.ftp_dropout(x, parts, 0.3, words, **{"site": 4, **other})
        assert abs(((parts != 0) == (y != 0)).double().mean().item() - (0.7 ** 2 + 0.3 ** 2)) < 0.02      # independent: 4.5 deviations are 0.009
    hole = x.clone()
    hole[y == 0] = math.nan
    F.ftp_dropout(hole, parts, 0.3, words, site=4)
    assert torch.equal(y, parts)                                        # whatever was dropped
    # the rate: 64000 draws of deviation 0.46 lie within 5 deviations of their mean
    assert abs((y == 0).double().mean().item() - 0.3) < 5 * 0.46 / math.sqrt(x.numel())


# ---- join -----------------------------------------------------------------------------------------------------------
JOIN = [(1, 1, 0, 0), (1, 64, 0, 0), (3, 7, 0, 0), (5, 40, 3, 1), (67, 96, 8, 0), (33, 257, 0, 0), (200, 1283, 0, 0), (9, 4096, 0, 0), (300, 512, 0, 8), (4, 8200, 0, 0), (3, 16384, 0, 0),
        (2, 12001, 1, 1), (70, 9000, 0, 0), (37, 768, 0, 0), (40, 1272, 0, 0), (21, 2560, 0, 0), (12, 3584, 16, 0), (9, 5120, 0, 0), (10, 6117, 1, 3), (7, 7168, 0, 0), (6, 8192, 0, 0)]
HOW = [dict(post="rms", pre="rms", gate="vector", p=0.1), dict(post="layer", pre="layer", gate=7, p=0.25, bias=1), dict(post="none", pre="layer", gate=None, p=0.0, bias=1),
       dict(post="rms", pre="none", gate=1, p=0.5), dict(post="layer", pre="rms", gate=50, p=0.0, bare=1), dict(post="none", pre="none", gate="vector", p=0.3),
       dict(post="layer", pre="layer", gate=None, p=0.0), dict(post="layer", pre="layer", gate="vector", p=0.1, bias=1),
       dict(post="none", pre="rms", gate=30, p=0.1), dict(post="none", pre="layer", gate="vector", p=0.2, bias=1), dict(post="layer", pre="rms", gate=9, p=0.1, bias=1)]


def join_case(rows, cols, gap, off, dt, how):
    """Options as the call takes them, and as the oracle does."""
    g = gen(rows, cols, str(dt), str(how))
    gate = how["gate"]
    gate_rows = gate if isinstance(gate, int) else 0
    own = dict(post=H.NORMS[how["post"]], pre=H.NORMS[how["pre"]], alpha=0.75, beta=1.5, gate_rows=gate_rows, dropout=how["p"], site=3, row0=5)
    ref = dict(post=how["post"], pre=how["pre"], alpha=0.75, beta=1.5, gate_rows=gate_rows, eps=1e-5)
    ref["eps"] = float(torch.tensor(1e-5, dtype=torch.float32))
    for name, on in (("w_post", how["post"] != "none" and not how.get("bare")), ("b_post", how["post"] != "none" and how.get("bias")),
                     ("w_pre", how["pre"] != "none" and not how.get("bare")), ("b_pre", how["pre"] != "none" and how.get("bias"))):
        own[name], ref[name] = vec(rnd(g, cols) + (1.0 if name[0] == "w" else 0.0) if on else None)
    if gate is None:
        own["gate"], ref["gate"] = None, None
    elif gate == "vector":
        own["gate"], ref["gate"] = vec(rnd(g, cols))
    else:
        m, ref["gate"] = on_gpu(rnd(g, -(-rows // gate), cols), dt, gap, off)
        own["gate"] = m.t
    own["rng"] = rng_of(77, 1 << 40) if how["p"] else None
    keep, f = H.keep_mask(rows, cols, how["p"], 77, 1 << 40, 3, 5)
    ref["mask"] = keep.double() * f if how["p"] else torch.ones(rows, cols, dtype=torch.float64)
    return g, own, ref


@pytest.mark.parametrize("rows,cols,gap,off", JOIN)
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("how", HOW, ids=lambda h: f"{h['post']}-{h['pre']}-{h['gate']}")
def test_join_forward_and_backward(rows, cols, gap, off, dt, how):
    g, own, ref = join_case(rows, cols, gap, off, dt, how)
    u, u64 = on_gpu(rnd(g, rows, cols) + 0.3, dt, gap, off)
    x, x64 = on_gpu(rnd(g, rows, cols, scale=2.0), dt, gap, off)
    s, y = Guarded(rows, cols, dt, gap, off), Guarded(rows, cols, dt, gap, off)
    stats = torch.full((4, rows), -7.0, device="cuda")
    pre = how["pre"] != "none"
    b_pre = own.pop("b_pre")
    F.ftp_join_forward(u.t, x.t, s.t, y.t if pre else None, b_pre=b_pre, eps=1e-5, stats=stats, **own)
    close(s.t, H.join_forward(u64, x64, ref), dt, "s")
    s64 = s.t.double().cpu()
    if pre:
        close(y.t, H.pre_forward(s64, ref), dt, "y")
    assert s.untouched() and y.untouched()
    for i, (kind, of) in enumerate(((how["post"], u64), (how["pre"], s64))):
        if kind == "none":
            assert bool((stats[2 * i:2 * i + 2] == -7.0).all())
            continue
        mean, r = H.moments(of, kind, ref["eps"])
        assert_within(stats[2 * i], mean[:, 0], 2 * H.SUM * H.U * of.abs().mean(1), "mean")
        assert_within(stats[2 * i + 1], r[:, 0], (2 * H.SUM * H.U + 8 * H.U * r[:, 0] ** 2 * of.abs().mean(1) ** 2) * r[:, 0], "1 / deviation")
    # backward
    dy, dy64 = on_gpu(rnd(g, rows, cols), dt, gap, off)
    ds, ds64 = on_gpu(rnd(g, rows, cols), dt, gap, off)
    du, dx = Guarded(rows, cols, dt, gap, off), Guarded(rows, cols, dt, gap, off)
    grads = {"d" + n: torch.full((cols,), -7.0, device="cuda") for n in ("w_post", "b_post", "w_pre", "b_pre") if (how["post"] if "post" in n else how["pre"]) != "none"}
    dgate = None
    if own["gate"] is not None:
        dgate = Guarded(own["gate"].shape[0], cols, dt, gap, off) if own["gate_rows"] else None
        grads["dgate"] = dgate.t if dgate else torch.full((cols,), -7.0, device="cuda")
    F.ftp_join_backward(u.t, s.t if pre else None, dy.t if pre else None, ds.t, stats, du=du.t, dx=dx.t, **grads, **own)
    want = H.join_backward(u64, s64, dy64, ds64, ref)
    for name, t in (("du", du.t), ("dx", dx.t)):
        close(t, want[name], dt, name)
    for name, t in grads.items():
        close(t, want[name], t.dtype, name)
    assert du.untouched() and dx.untouched() and (dgate is None or dgate.untouched())


@pytest.mark.parametrize("rows,cols,dt", [(5000, 72, BF), (3001, 520, BF), (1500, 2048, FP), (200, 4096, BF), (90, 6000, FP), (40000, 40, FP), (9500, 2052, FP)])
@pytest.mark.parametrize("gate", ["vector", 64, 1000])
def test_join_backward_over_many_rows(rows, cols, dt, gate):
    how = dict(post="rms", pre="layer", gate=gate, p=0.1, bias=1)
    g, own, ref = join_case(rows, cols, 0, 0, dt, how)
    own.pop("b_pre")
    u, u64 = on_gpu(rnd(g, rows, cols).abs(), dt)                       # one sign: sums grow with the rows
    s, s64 = on_gpu(rnd(g, rows, cols), dt)
    dy, dy64 = on_gpu(rnd(g, rows, cols).abs(), dt)
    stats = torch.zeros(4, rows, dtype=torch.float64)
    for i, (kind, of) in enumerate(((how["post"], u64), (how["pre"], s64))):
        mean, r = H.moments(of, kind, ref["eps"])
        stats[2 * i], stats[2 * i + 1] = mean[:, 0], r[:, 0]
    grads = {"d" + n: torch.empty(cols, device="cuda") for n in ("w_post", "b_post", "w_pre", "b_pre")}
    grads["dgate"] = torch.empty_like(own["gate"])
    du, dx = torch.empty_like(u.t), torch.empty_like(u.t)
    call = lambda: F.ftp_join_backward(u.t, s.t, dy.t, None, stats.float().cuda(), du=du, dx=dx, **grads, **own)  # noqa: E731
    call()
    want = H.join_backward(u64, s64, dy64, None, ref)
    for name, t in {**grads, "du": du, "dx": dx}.items():
        close(t, want[name], t.dtype, name)
    first = {n: t.clone() for n, t in grads.items()}
    call()
    assert all(torch.equal(first[n], t) for n, t in grads.items())


def test_a_norm_alone_and_a_branch_without_a_stream():
    g = gen("alone")
    for dt in (BF, FP):
        x, x64 = on_gpu(rnd(g, 30, 200), dt)
        w, w64 = vec(rnd(g, 200))
        y, stats = torch.empty_like(x.t), torch.empty(4, 30, device="cuda")
        F.ftp_join_forward(None, x.t, None, y, post=F.NORM_NONE, pre=F.NORM_RMS, w_pre=w, eps=1e-5, stats=stats)
        c = dict(pre="rms", post="none", eps=float(torch.tensor(1e-5)), w_pre=w64, b_pre=None, w_post=None, b_post=None, gate=None, gate_rows=0, alpha=1.0, beta=1.0,
                 mask=torch.ones(30, 200, dtype=torch.float64))
        close(y, H.pre_forward(x64, c), dt, "y")
        dx, dw = torch.empty_like(x.t), torch.empty(200, device="cuda")
        dy, dy64 = on_gpu(rnd(g, 30, 200), dt)
        F.ftp_join_backward(None, x.t, dy.t, None, stats, dx=dx, dw_pre=dw, post=F.NORM_NONE, pre=F.NORM_RMS, w_pre=w)
        want = H.join_backward(None, x64, dy64, None, c)
        close(dx, want["dx"], dt, "dx")
        close(dw, want["dw_pre"], FP, "dw_pre")
        s = torch.empty_like(x.t)
        F.ftp_join_forward(x.t, None, s, y, post=F.NORM_NONE, pre=F.NORM_RMS, w_pre=w, eps=1e-5)
        assert torch.equal(s, x.t)


def test_join_in_place_of_the_stream_and_of_its_gradient():
    g = gen("place")
    for dt in (BF, FP):
        u, x = (rnd(g, 50, 136).to(dt).cuda() for _ in range(2))
        s, y, y2, st = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty(4, 50, device="cuda")
        F.ftp_join_forward(u, x, s, y, stats=st)
        F.ftp_join_forward(u, x, x, y2)
        assert torch.equal(s, x) and torch.equal(y, y2)
        dy, ds = (rnd(g, 50, 136).to(dt).cuda() for _ in range(2))
        dx, du, du2 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
        F.ftp_join_backward(u, s, dy, ds, st, du=du, dx=dx)
        F.ftp_join_backward(u, s, dy, ds, st, du=du2, dx=ds)
        assert torch.equal(dx, ds) and torch.equal(du, du2)


def test_join_fused_mask_is_the_dropout_call_and_ignores_cuts():
    g = gen("mask")
    words = rng_of(3, 4)
    for cols in (264, 133):
        for dt in (BF, FP):
            u = rnd(g, 40, cols).to(dt).cuda()
            s, d = torch.empty_like(u), torch.empty_like(u)
            how = dict(post=F.NORM_NONE, pre=F.NORM_NONE, dropout=0.2, rng=words, site=11)
            F.ftp_join_forward(u, None, s, **how)
            F.ftp_dropout(u, d, 0.2, words, site=11)
            assert torch.equal(s, d)
            parts = torch.empty_like(u)
            for a, b in ((0, 1), (1, 33), (33, 40)):
                F.ftp_join_forward(u[a:b], None, parts[a:b], row0=a, **how)
            assert torch.equal(s, parts)


def test_join_gradients_match_differences():
    """Directional differences of a float64 form against the kernel's float gradients: error of the difference about 1e-8."""
    g = gen("diff")
    how = dict(post="layer", pre="rms", gate=3, p=0.25, bias=1)
    g, own, ref = join_case(10, 24, 0, 0, FP, how)
    own.pop("b_pre")
    vals = {"u": rnd(g, 10, 24), "x": rnd(g, 10, 24), **{k: ref[k] for k in ("w_post", "b_post", "w_pre", "b_pre", "gate") if ref[k] is not None}}
    vals = {k: v.float().double() for k, v in vals.items()}
    dy, ds = rnd(g, 10, 24).float().double(), rnd(g, 10, 24).float().double()

    def loss(v):
        c = {**ref, **{k: v[k] for k in v if k not in ("u", "x")}}
        s, _ = H.join_forward(v["u"], v["x"], c)
        return float((s * ds).sum() + (H.pre_forward(s, c)[0] * dy).sum())
    s64, _ = H.join_forward(vals["u"], vals["x"], {**ref, **{k: vals[k] for k in vals if k not in ("u", "x")}})
    stats = torch.cat([t[:, 0][None] for kind, of in (("layer", vals["u"]), ("rms", s64)) for t in H.moments(of, kind, ref["eps"])]).float().cuda()
    names = ["w_post", "b_post", "w_pre", "gate"]
    grads = {"d" + n: torch.empty_like(vals[n], dtype=FP, device="cuda") for n in names}
    du, dx = torch.empty(10, 24, device="cuda"), torch.empty(10, 24, device="cuda")
    F.ftp_join_backward(vals["u"].float().cuda(), s64.float().cuda(), dy.float().cuda(), ds.float().cuda(), stats, du=du, dx=dx, **grads, **own)
    for name, got in [("u", du), ("x", dx)] + [(n, grads["d" + n]) for n in names]:
        way = rnd(g, *vals[name].shape)
        e = 1e-5
        diff = (loss({**vals, name: vals[name] + e * way}) - loss({**vals, name: vals[name] - e * way})) / (2 * e)
        size = float((got.double().cpu() * way).abs().sum())
        assert abs(float((got.double().cpu() * way).sum()) - diff) < 1e-5 * size + 1e-6, name


def test_non_finite_tokens_stay_in_their_rows():
    for dt in (BF, FP):
        for cols in (64, 520, 77):
            u, x = torch.randn(9, cols, device="cuda").to(dt), torch.randn(9, cols, device="cuda").to(dt)
            u[2, 3], x[5, 1], u[7, 0] = math.nan, math.inf, math.inf
            s, y, st = torch.empty_like(u), torch.empty_like(u), torch.empty(4, 9, device="cuda")
            F.ftp_join_forward(u, x, s, y, post=F.NORM_LAYER, pre=F.NORM_LAYER, stats=st)
            bad = ~torch.isfinite(y).all(1)
            assert bad.nonzero()[:, 0].tolist() == [2, 5, 7]
            dy, du, dx = torch.randn_like(u), torch.empty_like(u), torch.empty_like(u)
            F.ftp_join_backward(u, s, dy, None, st, du=du, dx=dx, post=F.NORM_LAYER, pre=F.NORM_LAYER)
            assert [i for i in range(9) if not torch.isfinite(du[i]).all()] == [2, 5, 7]


def test_rows_of_one_value_and_of_zeros():
    for dt in (BF, FP):
        x = torch.zeros(4, 96, device="cuda", dtype=dt)
        x[1] = 3.0
        x[2, 5] = 1.0
        y = torch.empty_like(x)
        F.ftp_join_forward(None, x, None, y, post=F.NORM_NONE, pre=F.NORM_LAYER, eps=1e-5)
        assert not y[0].any() and not y[1].any() and bool(torch.isfinite(y).all())
        F.ftp_join_forward(None, x, None, y, post=F.NORM_NONE, pre=F.NORM_RMS, eps=0.0)
        assert bool(torch.isfinite(y[1:3]).all())


# ---- recurrence ----------------------------------------------------------------------------------------------------
def rec_inputs(g, rows, cols, dt, gap=0, off=0, coupled=True):
    f, f64 = on_gpu(rnd(g, rows, cols) + torch.linspace(0, 6, cols, dtype=torch.float64), dt, gap, off)
    v, v64 = on_gpu(rnd(g, rows, cols, scale=1.0 if coupled else 0.1), dt, gap, off)
    o, o64 = on_gpu(rnd(g, rows, cols, scale=1.5), dt, gap, off)
    return f, f64, v, v64, o, o64


REC = [(1, 1, 1, 0, 0), (3, 1, 64, 0, 0), (70, 1, 130, 0, 0), (2, 16, 33, 0, 0), (1, 17, 64, 0, 0), (2, 31, 65, 3, 1), (5, 100, 96, 2, 0), (1, 129, 200, 0, 0), (3, 257, 31, 1, 1), (1, 1000, 64, 0, 8),
       (1, 2500, 40, 0, 0), (2, 777, 300, 0, 0), (40, 40, 72, 0, 0), (300, 20, 64, 0, 0), (1, 3000, 33, 1, 1), (1, 2100, 66, 1, 0)]


@pytest.mark.parametrize("seqs,steps,cols,gap,off", REC)
@pytest.mark.parametrize("dt,name,coupled", [(BF, "silu", True), (FP, "gelu", True), (BF, None, False), (FP, None, False), (BF, "relu", True)])
def test_recurrence_forward_and_backward(seqs, steps, cols, gap, off, dt, name, coupled):
    g = gen(seqs, steps, cols, name)
    rows = seqs * steps
    f, f64, v, v64, o, o64 = rec_inputs(g, rows, cols, dt, gap, off, coupled)
    h0, h064 = vec(rnd(g, seqs, cols))
    three = lambda t: torch.as_strided(t, (seqs, steps, cols), (steps * t.stride(0), t.stride(0), 1), t.storage_offset()) if rows > 1 else t.view(1, 1, cols)  # noqa: E731
    y, h1 = Guarded(rows, cols, dt, gap, off), torch.empty(seqs, cols, device="cuda")
    states = torch.full((F.ftp_recurrence_states(rows, seqs), cols), -7.0, device="cuda")
    how = dict(coupled=coupled, act=ACTS[name] if name else 0)
    oo = three(o.t) if name else None
    F.ftp_recurrence_forward(three(f.t), three(v.t), three(y.t), o=oo, h0=h0, h1=h1, states=states, **how)
    dy, dy64 = on_gpu(rnd(g, rows, cols), dt, gap, off)
    dh1, dh164 = vec(rnd(g, seqs, cols))
    df, dv, do = (Guarded(rows, cols, dt, gap, off) for _ in range(3))
    dh0 = torch.empty(seqs, cols, device="cuda")
    F.ftp_recurrence_backward(three(f.t), three(v.t), three(dy.t), states, three(df.t), three(dv.t), o=oo, do=three(do.t) if name else None, dh1=dh1, dh0=dh0, **how)
    for b in range(seqs) if seqs < 10 else (0, 1, seqs // 2, seqs - 1):
        at = slice(b * steps, (b + 1) * steps)
        o1 = o64[at] if name else None
        hs, es, ys, ey = H.recurrence(f64[at], v64[at], o1, h064[b], name, coupled, dt)
        close(y.t[at], (ys, ey), dt, f"y of {b}")
        close(h1[b], (hs[-1], es[-1]), FP, f"h1 of {b}")
        kept = states[b * steps // 16 + b:][:-(-steps // 16)]
        close(kept[0], (h064[b], 0 * h064[b]), FP, "first state")
        close(kept[1:], (hs[15:steps - 1:16], es[15:steps - 1:16]), FP, f"states of {b}")
        want = H.recurrence_backward(f64[at], v64[at], o1, h064[b], dy64[at], dh164[b], name, coupled, dt)
        close(df.t[at], want["df"], dt, f"df of {b}")
        close(dv.t[at], want["dv"], dt, f"dv of {b}")
        if name:
            close(do.t[at], want["do"], dt, f"do of {b}")
        close(dh0[b], want["dh0"], FP, f"dh0 of {b}")
    assert y.untouched() and df.untouched() and dv.untouched() and do.untouched()


@pytest.mark.parametrize("lengths,cols", [([5, 0, 1, 33, 700, 16, 0, 17, 129], 70), ([0, 0], 8), ([1500, 3, 2], 64), ([2] * 50, 33), ([1, 0, 1], 5)])
@pytest.mark.parametrize("dt", [BF, FP])
def test_recurrence_over_packed_sequences(lengths, cols, dt):
    g = gen("packed", str(lengths))
    used = sum(lengths)
    rows, seqs = used + 5, len(lengths)                                  # rows behind the last sequence
    f, f64, v, v64, o, o64 = rec_inputs(g, rows, cols, dt)
    h0, h064 = vec(rnd(g, seqs, cols))
    off = torch.tensor([0] + torch.tensor(lengths).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
    y, df, dv, do = (torch.full_like(f.t, -7.0) for _ in range(4))
    h1, dh0 = torch.empty_like(h0), torch.empty_like(h0)
    states = torch.full((F.ftp_recurrence_states(rows, seqs), cols), -7.0, device="cuda")
    how = dict(act=F.ACT_SILU, offsets=off, max_len=max(max(lengths), 1))
    F.ftp_recurrence_forward(f.t, v.t, y, o=o.t, h0=h0, h1=h1, states=states, **how)
    dy, dy64 = on_gpu(rnd(g, rows, cols), dt)
    F.ftp_recurrence_backward(f.t, v.t, dy.t, states, df, dv, o=o.t, do=do, dh0=dh0, **how)
    a = 0
    for b, n in enumerate(lengths):
        at = slice(a, a + n)
        hs, es, ys, ey = H.recurrence(f64[at], v64[at], o64[at], h064[b], "silu", True, dt)
        want = H.recurrence_backward(f64[at], v64[at], o64[at], h064[b], dy64[at], 0 * h064[b], "silu", True, dt)
        close(h1[b], (hs[-1], es[-1]) if n else (h064[b], 0 * h064[b]), FP, "h1")
        close(dh0[b], want["dh0"], FP, "dh0")
        for name, t, pair in (("y", y, (ys, ey)), ("df", df, want["df"]), ("dv", dv, want["dv"]), ("do", do, want["do"])):
            close(t[at], pair, dt, f"{name} of {b}")
        a += n
    for t in (y, df, dv, do):
        assert bool((t[used:] == -7.0).all())


def test_recurrence_offsets_beyond_the_rows_and_longer_sequences_are_cut_off():
    f, v, o = (torch.randn(40, 64, device="cuda") for _ in range(3))
    for bad, max_len in (([-5, 20, 90], 40), ([0, 30, 10], 40), ([10, 35, 40], 8), ([50, 60, 70], 40)):
        y = torch.full_like(f, -7.0)
        states = torch.full((F.ftp_recurrence_states(40, 2), 64), -7.0, device="cuda")
        F.ftp_recurrence_forward(f, v, y, o=o, states=states, offsets=torch.tensor(bad, dtype=torch.int32, device="cuda"), max_len=max_len)
        inside = torch.zeros(40, dtype=torch.bool)
        for a, b in zip(bad, bad[1:]):
            a = min(max(a, 0), 40)
            b = min(max(b, a), 40)
            inside[a:min(b, a + max_len)] = True
        assert bool((y[~inside.cuda()] == -7.0).all()) and bool(torch.isfinite(y).all())


def test_recurrence_steps_continue_a_sequence_in_place():
    """A prompt, then token by token with the state updated in place, equals the whole sequence (and a time-major batch is one
    sequence of all channels)."""
    g = gen("steps")
    for dt in (BF, FP):
        f, v, o = (rnd(g, 3, 40, 72).to(dt).cuda() for _ in range(3))
        y, h1 = torch.empty_like(f), torch.empty(3, 72, device="cuda")
        F.ftp_recurrence_forward(f, v, y, o=o, h1=h1)
        got, h = torch.empty_like(f), torch.empty(3, 72, device="cuda")
        part = lambda a, b: (f[:, a:b].contiguous(), v[:, a:b].contiguous(), o[:, a:b].contiguous())  # noqa: E731
        for i, (a, b) in enumerate([(0, 33)] + [(t, t + 1) for t in range(33, 40)]):
            ff, vv, oo = part(a, b)
            yy = torch.empty_like(ff)
            F.ftp_recurrence_forward(ff, vv, yy, o=oo, h0=h if i else None, h1=h)
            got[:, a:b] = yy
        # the state passes through the same float operations a step at a time; the joined runs differ by float roundings
        rel = 2.0 ** -7 if dt is BF else 2.0 ** -18
        assert torch.allclose(got.float(), y.float(), rtol=rel, atol=rel) and torch.allclose(h, h1, rtol=2.0 ** -18, atol=2.0 ** -18)
        major = lambda t: t.transpose(0, 1).contiguous().view(40, 3 * 72)  # noqa: E731
        ym = torch.empty(40, 3 * 72, device="cuda", dtype=dt)
        F.ftp_recurrence_forward(major(f), major(v), ym, o=major(o))
        assert torch.equal(ym.view(40, 3, 72).transpose(0, 1), y)
        one = f[:, 5:6]                                                  # one step of a longer tensor: the gap between sequences is the pitch
        y1, y2 = torch.empty_like(one.contiguous()), torch.empty_like(one.contiguous())
        F.ftp_recurrence_forward(one, v[:, 5:6], y1, o=o[:, 5:6], h0=h)
        F.ftp_recurrence_forward(one.contiguous(), v[:, 5:6].contiguous(), y2, o=o[:, 5:6].contiguous(), h0=h)
        assert torch.equal(y1, y2)


def test_recurrence_extreme_gates():
    for dt in (BF, FP):
        f = torch.zeros(40, 6, device="cuda", dtype=dt)
        f[:, 0], f[:, 1], f[:, 2], f[:, 3], f[5, 4], f[5, 5] = math.inf, -math.inf, 200.0, -200.0, math.nan, -math.inf
        v = torch.randn(40, 6, device="cuda").to(dt)
        y, h1 = torch.empty_like(f), torch.empty(1, 6, device="cuda")
        F.ftp_recurrence_forward(f, v, y, h0=torch.full((1, 6), 2.0, device="cuda"), h1=h1)
        assert bool((y[:, 0] == 2).all()) and bool((y[:, 2] == 2).all()) and torch.equal(y[:, 1], v[:, 1]) and torch.equal(y[:, 3], v[:, 3])
        assert torch.isfinite(y[:5, 4]).all() and torch.isnan(y[5:, 4]).all() and y[5, 5] == v[5, 5] and torch.isfinite(y[:, 5]).all()


def test_recurrence_gradients_match_differences():
    g = gen("rec-diff")
    n, c = 50, 6
    vals = {k: rnd(g, n, c).float().double() for k in ("f", "v", "o")}
    vals["h0"] = rnd(g, c).float().double()
    dy, dh1 = rnd(g, n, c).float().double(), rnd(g, c).float().double()

    def loss(z):
        hs, _, ys, _ = H.recurrence(z["f"], z["v"], z["o"], z["h0"], "silu", True, FP)
        return float((ys * dy).sum() + (hs[-1] * dh1).sum())
    gpu = {k: t.float().cuda() for k, t in vals.items()}
    y, states = torch.empty(n, c, device="cuda"), torch.empty(F.ftp_recurrence_states(n, 1), c, device="cuda")
    F.ftp_recurrence_forward(gpu["f"], gpu["v"], y, o=gpu["o"], h0=gpu["h0"], states=states)
    df, dv, do, dh0 = (torch.empty_like(gpu[k]) for k in ("f", "v", "o", "h0"))
    F.ftp_recurrence_backward(gpu["f"], gpu["v"], dy.float().cuda(), states, df, dv, o=gpu["o"], do=do, dh1=dh1.float().cuda(), dh0=dh0)
    for name, got in (("f", df), ("v", dv), ("o", do), ("h0", dh0)):
        way = rnd(g, *vals[name].shape)
        e = 1e-5
        diff = (loss({**vals, name: vals[name] + e * way}) - loss({**vals, name: vals[name] - e * way})) / (2 * e)
        size = float((got.double().cpu() * way).abs().sum())
        assert abs(float((got.double().cpu() * way).sum()) - diff) < 1e-5 * size + 1e-6, name


# ---- log probabilities ----------------------------------------------------------------------------------------------
LOGP = [(1, 1, 0, 0), (3, 2, 0, 0), (5, 7, 0, 0), (2, 33, 3, 1), (7, 100, 0, 0), (130, 129, 1, 0), (3, 1000, 0, 3), (2, 5001, 0, 0), (1, 32000, 0, 0), (20, 50021, 3, 1), (400, 3001, 0, 0)]


def logits_of(g, rows, vocab, dt, gap=0, off=0, masked=False):
    z = rnd(g, rows, vocab, scale=2.0)
    if masked and vocab > 4:
        z[:, ::3] = -math.inf
    return on_gpu(z, dt, gap, off)


def top_of(x64, k):
    order = sorted(range(x64.shape[0]), key=lambda c: (-float(x64[c]), c))
    return order[:k]


@pytest.mark.parametrize("rows,vocab,gap,off", LOGP)
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("k,scale,masked", [(0, 1.0, False), (1, 1.5, True), (20, 0.7, False), (32, 1.0, True)])
def test_logprob_forward_and_backward(rows, vocab, gap, off, dt, k, scale, masked):
    g = gen(rows, vocab, k, str(dt))
    scale = float(torch.tensor(scale, dtype=torch.float32))
    k = min(k, vocab)
    x, x64 = logits_of(g, rows, vocab, dt, gap, off, masked)
    t = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    if rows > 2:
        t[1], t[2] = -1, vocab                                           # no target
    f32 = lambda *s: torch.full(s, -7.0, device="cuda")  # noqa: E731
    logp, ent, lse, tl = f32(rows), f32(rows), f32(rows, 2), f32(rows, k) if k else None
    top = torch.full((rows, k), -7, dtype=torch.int32, device="cuda") if k else None
    F.ftp_logprob_forward(x.t, t.cuda(), logp, entropy=ent, lse=lse, top=top, top_logp=tl, scale=scale)
    r_logp, r_ent, r_lse, lp, e1, e2 = H.logprob(x64, t, scale)
    fin = torch.isfinite(r_logp)
    assert bool((logp.cpu()[~fin] == -math.inf).all())
    assert_within(logp.cpu()[fin], r_logp[fin], e1[fin], "logp")
    assert_within(ent, r_ent, e2, "entropy")
    assert torch.equal(lse[:, 0].double().cpu(), r_lse[:, 0])
    assert_within(lse[:, 1], r_lse[:, 1], e1, "log sum")
    if k:
        for r in list(range(min(rows, 6))) + [rows - 1]:
            want = top_of(x64[r], k)
            assert top[r].tolist() == want, r
            ref = lp[r][want]
            ok = torch.isfinite(ref)
            assert bool((tl[r].cpu()[~ok] == -math.inf).all())
            assert_within(tl[r].cpu()[ok], ref[ok], e1[r] + 4 * H.U * ref[ok].abs(), "top logp")
    bare = f32(rows)
    F.ftp_logprob_forward(x.t, t.cuda(), bare, scale=scale)              # without the entropy, the same sums
    assert torch.equal(bare, logp)
    dl, dl64 = vec(rnd(g, rows))
    dh, dh64 = vec(rnd(g, rows))
    for a, b in ((dl, None), (None, dh), (dl, dh)):
        d = Guarded(rows, vocab, dt, gap, off)
        F.ftp_logprob_backward(x.t, t.cuda(), lse, a, d.t, entropy=ent, dentropy=b, scale=scale)
        close(d.t, H.logprob_backward(x64, t, scale, dl64 if a is not None else None, dh64 if b is not None else None), dt, "dlogits")
        assert d.untouched()
    other = Guarded(rows, vocab, dt, gap + 1, off + 1)                   # rows that lie otherwise than the logits'
    F.ftp_logprob_backward(x.t, t.cuda(), lse, dl, other.t, entropy=ent, dentropy=dh, scale=scale)
    assert torch.equal(other.t, d.t) and other.untouched()
    F.ftp_logprob_backward(x.t, t.cuda(), lse, dl, x.t, entropy=ent, dentropy=dh, scale=scale)
    assert torch.equal(x.t, d.t) and x.untouched()                       # in place


@pytest.mark.parametrize("vocab", [40, 9000, 70000])
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("rows", [1, 3, 500])
def test_logprob_masks_ties_and_rows_of_nothing(vocab, dt, rows):
    low = torch.finfo(dt).min
    x = torch.zeros(6, vocab, dtype=torch.float64)                       # 0: all alike
    x[1] = -math.inf                                                     # nothing
    x[2] = low                                                           # nothing but the lowest value
    x[3] = -math.inf
    x[3, vocab // 2] = 1.0                                               # one token
    x[4] = low
    x[4, -1], x[4, 0] = -5.0, -5.0                                       # two tokens
    x[5] = torch.arange(vocab) % 4 == 3                                  # many equal
    x[5, 7] = -0.0
    x = x[torch.arange(rows) % 6] if rows > 3 else x[[5, 0, 2][:rows]] if rows > 1 else x[5:6]
    xd, x64 = x.to(dt).cuda(), x.to(dt).double()
    t = torch.full((rows,), vocab // 2, dtype=torch.int32)
    k = 32
    logp, ent, lse, tl = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda"), \
        torch.empty(rows, k, device="cuda")
    top = torch.empty(rows, k, dtype=torch.int32, device="cuda")
    F.ftp_logprob_forward(xd, t.cuda(), logp, entropy=ent, lse=lse, top=top, top_logp=tl)
    r_logp, r_ent, r_lse, lp, e1, e2 = H.logprob(x64, t, 1.0)
    fin = torch.isfinite(r_logp)
    assert bool((logp.cpu()[~fin] == -math.inf).all())
    # next to the lowest value the rest of the row is infinitely far: magnitudes of 1e38 do not enter the bound
    assert_within(logp.cpu()[fin], r_logp[fin], e1[fin].clamp(max=1e-3), "logp")
    assert_within(ent, r_ent, e2, "entropy")
    for r in range(min(rows, 6)):
        assert top[r].tolist() == top_of(x64[r], k), r
    d, dl, dh = torch.empty_like(xd), torch.ones(rows, device="cuda"), torch.ones(rows, device="cuda")
    F.ftp_logprob_backward(xd, t.cuda(), lse, dl, d, entropy=ent, dentropy=dh)
    close(d, H.logprob_backward(x64, t, 1.0, dl.double().cpu(), dh.double().cpu()), dt, "dlogits")


@pytest.mark.parametrize("rows,vocab", [(592, 1), (593, 37), (595, 1025), (2371, 1500), (2370, 4500), (9475, 90)])
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("k", [1, 32])
def test_logprob_many_short_rows(rows, vocab, dt, k):
    """Rows enough to fill the GPU, of few tokens: random ones among masked ones, ties and rows of nothing, next to one another."""
    g = gen("lp-short", rows, vocab, k, str(dt))
    z = rnd(g, rows, vocab, scale=2.0)
    z[1::5, ::2] = -math.inf
    z[2::5] = 0.5
    z[3::25] = -math.inf
    z[4::5] = (torch.arange(vocab) % 4 == 1).double()
    x, x64 = on_gpu(z, dt, 1, 1)
    k, scale = min(k, vocab), 1.25
    t = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    f32 = lambda *s: torch.full(s, -7.0, device="cuda")  # noqa: E731
    logp, bare, ent, lse, tl = f32(rows), f32(rows), f32(rows), f32(rows, 2), f32(rows, k)
    top = torch.full((rows, k), -7, dtype=torch.int32, device="cuda")
    F.ftp_logprob_forward(x.t, t.cuda(), logp, entropy=ent, lse=lse, top=top, top_logp=tl, scale=scale)
    F.ftp_logprob_forward(x.t, t.cuda(), bare, scale=scale)
    assert torch.equal(bare, logp)
    r_logp, r_ent, r_lse, lp, e1, e2 = H.logprob(x64, t, scale)
    fin = torch.isfinite(r_logp)
    assert bool((logp.cpu()[~fin] == -math.inf).all())
    assert_within(logp.cpu()[fin], r_logp[fin], e1[fin], "logp")
    assert_within(ent, r_ent, e2, "entropy")
    assert torch.equal(lse[:, 0].double().cpu(), r_lse[:, 0])
    want = torch.sort(x64, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(top.cpu().long(), want)
    ref = lp.gather(1, want)
    ok = torch.isfinite(ref)
    assert bool((tl.cpu()[~ok] == -math.inf).all())
    assert_within(tl.cpu()[ok], ref[ok], (e1[:, None] + 4 * H.U * ref.nan_to_num(0, 0, 0).abs())[ok], "top logp")


def test_logprob_rows_with_nan_and_infinity():
    for dt in (BF, FP):
        for vocab in (50, 20001):
            x = torch.randn(5, vocab, device="cuda").to(dt)
            x[1, 3], x[2, vocab - 1], x[4] = math.nan, math.inf, -math.nan
            t = torch.zeros(5, dtype=torch.int32, device="cuda")
            logp, ent, lse, top = torch.empty(5, device="cuda"), torch.empty(5, device="cuda"), torch.empty(5, 2, device="cuda"), torch.empty(5, 9, dtype=torch.int32, device="cuda")
            F.ftp_logprob_forward(x, t, logp, entropy=ent, lse=lse, top=top)
            for r in range(5):
                assert bool(torch.isnan(logp[r])) == (r in (1, 2, 4)) and bool(torch.isnan(ent[r])) == (r in (1, 2, 4))
            assert bool(((top >= 0) & (top < vocab)).all())
            d = torch.empty_like(x)
            F.ftp_logprob_backward(x, t, lse, torch.ones(5, device="cuda"), d)
            for r in range(5):
                assert bool(torch.isnan(d[r]).any()) == (r in (1, 2, 4))


def test_logprob_gradients_match_differences():
    g = gen("lp-diff")
    x = rnd(g, 4, 30).float().double()
    t = torch.tensor([1, 29, -1, 0], dtype=torch.int32)
    dl, dh = rnd(g, 4).float().double(), rnd(g, 4).float().double()
    loss = lambda v: float((H.logprob(v, t, 1.25)[0] * dl + H.logprob(v, t, 1.25)[1] * dh).sum())  # noqa: E731
    xd = x.float().cuda()
    logp, ent, lse, d = torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty(4, 2, device="cuda"), torch.empty_like(xd)
    F.ftp_logprob_forward(xd, t.cuda(), logp, entropy=ent, lse=lse, scale=1.25)
    F.ftp_logprob_backward(xd, t.cuda(), lse, dl.float().cuda(), d, entropy=ent, dentropy=dh.float().cuda(), scale=1.25)
    way, e = rnd(g, 4, 30), 1e-5
    diff = (loss(x + e * way) - loss(x - e * way)) / (2 * e)
    assert abs(float((d.double().cpu() * way).sum()) - diff) < 1e-5 * float((d.double().cpu() * way).abs().sum()) + 1e-6


# ---- all of them, with the products ---------------------------------------------------------------------------------
class Net:
    """One block of a language model and its head, as a program strings it together: norm, projections, recurrence, projection, join
    with dropout, gated feed-forward product, join, logits, log probabilities; and back."""

    def __init__(self, g, rows, seqs, d, f, vocab, dt):
        self.dt, self.rows, self.seqs = dt, rows, seqs
        w = lambda a, b: (rnd(g, a, b) * a ** -0.5).to(dt).cuda()  # noqa: E731
        self.w = {"f": w(d, d), "v": w(d, d), "o": w(d, d), "out": w(d, d), "gate": w(d, f), "up": w(d, f), "down": w(f, d), "head": w(d, vocab)}
        self.n = {k: (1.0 + 0.1 * rnd(g, d)).float().cuda() for k in ("in", "post1", "mid", "post2", "last")}
        e = lambda *s: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
        r = rows
        self.b = {k: e(r, d) for k in ("y0", "f", "v", "o", "h", "a", "s1", "y1", "m", "s2", "y2", "dx", "dy2", "ds2", "dm", "dy1", "ds1", "da", "dh", "df", "dv", "do", "dy0")}
        self.b.update(p=e(2, r, f), hh=e(r, f), dhh=e(r, f), z=e(r, vocab), dz=e(r, vocab))
        self.st = [torch.empty(4, r, device="cuda") for _ in range(3)]
        self.states = torch.empty(F.ftp_recurrence_states(r, seqs), d, device="cuda")
        self.logp, self.ent, self.lse = torch.empty(r, device="cuda"), torch.empty(r, device="cuda"), torch.empty(r, 2, device="cuda")
        self.gw = {k: torch.empty_like(t) for k, t in self.w.items()}
        self.gn = {k: torch.empty_like(t) for k, t in self.n.items()}
        self.rng = rng_of(5, 0)
        self.dl = torch.full((r,), -1.0 / r, device="cuda")

    def step(self, x, t):
        b, w, n = self.b, self.w, self.n
        seq = lambda k: b[k].view(self.seqs, -1, b[k].shape[1])  # noqa: E731
        how1 = dict(w_post=n["post1"], w_pre=n["mid"], beta=0.5, dropout=0.25, rng=self.rng, site=0)
        how2 = dict(w_post=n["post2"], w_pre=n["last"], pre=F.NORM_LAYER, dropout=0.25, rng=self.rng, site=1)
        F.ftp_join_forward(None, x, None, b["y0"], post=F.NORM_NONE, w_pre=n["in"], stats=self.st[0])
        for k in "fvo":
            F.ftp_linear_forward(b["y0"], w[k], b[k])
        F.ftp_recurrence_forward(seq("f"), seq("v"), seq("h"), o=seq("o"), states=self.states)
        F.ftp_linear_forward(b["h"], w["out"], b["a"])
        F.ftp_join_forward(b["a"], x, b["s1"], b["y1"], stats=self.st[1], **how1)
        F.ftp_gated_forward(b["y1"], w["gate"], w["up"], b["hh"], stash=b["p"])
        F.ftp_linear_forward(b["hh"], w["down"], b["m"])
        F.ftp_join_forward(b["m"], b["s1"], b["s2"], b["y2"], stats=self.st[2], **how2)
        F.ftp_linear_forward(b["y2"], w["head"], b["z"])
        F.ftp_logprob_forward(b["z"], t, self.logp, entropy=self.ent, lse=self.lse)
        g, gn = self.gw, self.gn
        F.ftp_logprob_backward(b["z"], t, self.lse, self.dl, b["dz"])
        F.ftp_linear_backward(b["y2"], w["head"], b["dz"], dx=b["dy2"], dw=g["head"])
        F.ftp_join_backward(b["m"], b["s2"], b["dy2"], None, self.st[2], du=b["dm"], dx=b["ds2"], dw_post=gn["post2"], dw_pre=gn["last"], **how2)
        F.ftp_linear_backward(b["hh"], w["down"], b["dm"], dx=b["dhh"], dw=g["down"])
        F.ftp_gated_backward(b["y1"], w["gate"], w["up"], b["dhh"], dx=b["dy1"], dw_gate=g["gate"], dw_up=g["up"], stash=b["p"])
        F.ftp_join_backward(b["a"], b["s1"], b["dy1"], b["ds2"], self.st[1], du=b["da"], dx=b["ds1"], dw_post=gn["post1"], dw_pre=gn["mid"], **how1)
        F.ftp_linear_backward(b["h"], w["out"], b["da"], dx=b["dh"], dw=g["out"])
        F.ftp_recurrence_backward(seq("f"), seq("v"), seq("dh"), self.states, seq("df"), seq("dv"), o=seq("o"), do=seq("do"))
        F.ftp_linear_backward(b["y0"], w["f"], b["df"], dx=b["dy0"], dw=g["f"])
        for k in "vo":
            F.ftp_linear_backward(b["y0"], w[k], b["d" + k], dx=b["dy0"], dw=g[k], dx_addend=b["dy0"])
        F.ftp_join_backward(None, x, b["dy0"], b["ds1"], self.st[0], dx=b["dx"], dw_pre=gn["in"], post=F.NORM_NONE, w_pre=n["in"])


def plain_net(net, x, t, masks):
    """The same loss by autograd in float64."""
    p = {k: v.double().cpu().requires_grad_() for k, v in net.w.items()}
    n = {k: v.double().cpu().requires_grad_() for k, v in net.n.items()}
    x = x.double().cpu().requires_grad_()
    rms = lambda v, w: v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6) * w  # noqa: E731
    y0 = rms(x, n["in"])
    f, v, o = y0 @ p["f"], y0 @ p["v"], y0 @ p["o"]
    a = torch.sigmoid(f).view(net.seqs, -1, f.shape[1])
    bb = (torch.sigmoid(-f) * v).view_as(a)
    h, hs = torch.zeros_like(a[:, 0]), []
    for i in range(a.shape[1]):
        h = a[:, i] * h + bb[:, i]
        hs.append(h)
    y = torch.stack(hs, 1).reshape_as(f) * o * torch.sigmoid(o)
    s1 = x + 0.5 * masks[0] * rms(y @ p["out"], n["post1"])
    y1 = rms(s1, n["mid"])
    g = y1 @ p["gate"]
    m = (g * torch.sigmoid(g) * (y1 @ p["up"])) @ p["down"]
    s2 = s1 + masks[1] * rms(m, n["post2"])
    c = s2 - s2.mean(1, keepdim=True)
    y2 = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-6) * n["last"]
    lp = torch.log_softmax(y2 @ p["head"], 1).gather(1, t.cpu().long()[:, None])[:, 0]
    (-lp.mean()).backward()
    return lp.detach(), {k: v.grad for k, v in p.items()}, {k: v.grad for k, v in n.items()}, x.grad


@pytest.mark.parametrize("rows,seqs,d,f,vocab", [(96, 2, 64, 128, 300), (130, 5, 72, 100, 77)])
def test_a_block_and_its_head_train_as_in_64_bits(rows, seqs, d, f, vocab):
    g = gen("net", rows)
    net = Net(g, rows, seqs, d, f, vocab, FP)
    x = rnd(g, rows, d).float().cuda()
    t = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32).cuda()
    net.step(x, t)
    masks = [k.double() * c for k, c in (H.keep_mask(rows, d, 0.25, 5, 0, site) for site in (0, 1))]
    lp, gw, gn, gx = plain_net(net, x, t, masks)
    # float tensors throughout: some 20 operators of 1e-6 each on values of size 1, gradients relative to their largest
    assert (net.logp.double().cpu() - lp).abs().max() < 2e-5 * max(1.0, float(lp.abs().max()))
    for name, got, want in [("x", net.b["dx"], gx)] + [(k, net.gw[k], gw[k]) for k in gw] + [(k, net.gn[k], gn[k]) for k in gn]:
        assert (got.double().cpu() - want).abs().max() < 1e-4 * float(want.abs().max()), name


@pytest.mark.parametrize("dt", [BF, FP])
def test_captured_block_replays_with_new_inputs_and_a_new_mask(dt):
    g = gen("graph")
    net = Net(g, 96, 2, 64, 128, 304, dt)
    x, t = rnd(g, 96, 64).to(dt).cuda(), torch.randint(0, 304, (96,), generator=g, dtype=torch.int32).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        net.step(x, t)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.step(x, t)
    results = []
    for step in (1, 2, 2):
        x.copy_(rnd(gen("x", step), 96, 64).to(dt))
        net.rng[1] = step
        graph.replay()
        torch.cuda.synchronize()
        results.append([net.logp.clone(), net.b["dx"].clone(), net.gw["f"].clone(), net.gn["post1"].clone()])
    for a, b in zip(results[1], results[2]):
        assert torch.equal(a, b)
    assert not torch.equal(results[0][0], results[1][0])
    net.rng[1] = 1
    x.copy_(rnd(gen("x", 1), 96, 64).to(dt))
    net.step(x, t)
    for a, b in zip(results[0], [net.logp, net.b["dx"], net.gw["f"], net.gn["post1"]]):
        assert torch.equal(a, b)


def test_calls_on_other_streams_and_threads_at_once():
    g = gen("threads")
    nets = [Net(gen("threads", i), 130, 2, 72, 128, 304, BF) for i in range(3)]
    xs = [rnd(g, 130, 72).to(BF).cuda() for _ in nets]
    ts = [torch.randint(0, 304, (130,), generator=g, dtype=torch.int32).cuda() for _ in nets]
    want = []
    for net, x, t in zip(nets, xs, ts):
        net.step(x, t)
        want.append([net.logp.clone(), net.b["dx"].clone(), net.gn["post2"].clone()])
    torch.cuda.synchronize()
    errors = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(5):
                    nets[i].step(xs[i], ts[i])
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(3)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not errors
    for net, w in zip(nets, want):
        assert torch.equal(net.logp, w[0]) and torch.equal(net.b["dx"], w[1]) and torch.equal(net.gn["post2"], w[2])


def test_first_calls_of_a_process_may_be_captured():
    code = """
import torch, paper_2110_02781_b200 as F
dev = dict(device="cuda")
f, v, o, y = (torch.randn(2, 300, 64, **dev).bfloat16() for _ in range(4))
states, dy = torch.empty(F.ftp_recurrence_states(600, 2), 64, **dev), torch.randn(2, 300, 64, **dev).bfloat16()
df, dv, do = (torch.empty_like(f) for _ in range(3))
x, s, z, st = torch.randn(600, 4096, **dev).bfloat16(), torch.empty(600, 4096, **dev).bfloat16(), torch.empty(600, 4096, **dev).bfloat16(), torch.empty(4, 600, **dev)
w, du, dx, dw, dw2 = torch.ones(4096, **dev), torch.empty_like(x), torch.empty_like(x), torch.empty(4096, **dev), torch.empty(4096, **dev)
t, lp, lse, top = torch.zeros(600, dtype=torch.int32, **dev), torch.empty(600, **dev), torch.empty(600, 2, **dev), torch.empty(600, 5, dtype=torch.int32, **dev)
rng = torch.tensor([1, 2], dtype=torch.int64, **dev)
def step():
    F.ftp_recurrence_forward(f, v, y, o=o, states=states)
    F.ftp_recurrence_backward(f, v, dy, states, df, dv, o=o, do=do)
    F.ftp_join_forward(x, x, s, z, w_post=w, w_pre=w, dropout=0.1, rng=rng, stats=st)
    F.ftp_join_backward(x, s, z, x, st, du=du, dx=dx, dw_post=dw, dw_pre=dw2, w_post=w, w_pre=w, dropout=0.1, rng=rng)
    F.ftp_logprob_forward(s, t, lp, lse=lse, top=top)
    F.ftp_logprob_backward(s, t, lse, lp, du)
    F.ftp_dropout(x, dx, 0.3, rng)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    step()
g.replay()
torch.cuda.synchronize()
out = [y, df, do, dw, dw2, lp, top, du, dx]
a = [q.clone() for q in out]
step()
assert all(torch.equal(p, q) for p, q in zip(a, out))
F.ftp_check_op_status()
print("same")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=str(Path(__file__).parent.parent))
    assert r.returncode == 0 and "same" in r.stdout, r.stdout + r.stderr


def test_no_rows():
    for dt in (BF, FP):
        e = lambda *s: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
        F.ftp_dropout(e(0, 8), e(0, 8), 0.5, rng_of(1, 1))
        F.ftp_join_forward(e(0, 8), e(0, 8), e(0, 8), e(0, 8))
        dw, db = torch.ones(8, device="cuda"), torch.ones(8, device="cuda")
        F.ftp_join_backward(e(0, 8), e(0, 8), e(0, 8), None, torch.empty(4, 0, device="cuda"), du=e(0, 8), dx=e(0, 8), dw_post=dw, db_pre=db)
        assert not dw.any() and not db.any()
        h0, h1 = torch.randn(3, 8, device="cuda"), torch.empty(3, 8, device="cuda")
        F.ftp_recurrence_forward(e(3, 0, 8), e(3, 0, 8), e(3, 0, 8), h0=h0, h1=h1)
        assert torch.equal(h0, h1)
        states = torch.empty(3, 8, device="cuda")
        F.ftp_recurrence_backward(e(3, 0, 8), e(3, 0, 8), e(3, 0, 8), states, e(3, 0, 8), e(3, 0, 8), dh1=h0, dh0=h1.zero_())
        assert torch.equal(h0, h1)
        F.ftp_recurrence_forward(e(0, 5, 8), e(0, 5, 8), e(0, 5, 8))
        none = torch.empty(0, device="cuda")
        F.ftp_logprob_forward(e(0, 8), torch.empty(0, dtype=torch.int32, device="cuda"), none)


def test_wide_offsets():
    """Rows whose elements lie beyond 2^31."""
    rows, cols, ld = 5, 96, 600_000_000
    buf = torch.zeros((rows - 1) * ld + cols, dtype=BF, device="cuda")
    far = torch.as_strided(buf, (rows, cols), (ld, 1))
    near = torch.randn(rows, cols, device="cuda").to(BF)
    far.copy_(near)
    a, b, y = torch.empty_like(near), torch.empty_like(near), torch.empty_like(near)
    F.ftp_dropout(far, a, 0.25, rng_of(1, 2))
    F.ftp_dropout(near, b, 0.25, rng_of(1, 2))
    assert torch.equal(a, b)
    F.ftp_join_forward(far, far, a, y)
    F.ftp_join_forward(near, near, b, z := torch.empty_like(near))
    assert torch.equal(a, b) and torch.equal(y, z)
    F.ftp_recurrence_forward(far, far, a)
    F.ftp_recurrence_forward(near, near, b)
    assert torch.equal(a, b)
    t = torch.arange(rows, dtype=torch.int32, device="cuda")
    la, lb = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    F.ftp_logprob_forward(far, t, la)
    F.ftp_logprob_forward(near, t, lb)
    assert torch.equal(la, lb)
    F.ftp_dropout(near, far, 0.25, rng_of(1, 2))
    F.ftp_dropout(near, b, 0.25, rng_of(1, 2))
    assert torch.equal(far, b)


def test_refusals():
    bf = lambda *s: torch.zeros(*s, dtype=BF, device="cuda")  # noqa: E731
    f32 = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    words, i32 = rng_of(1, 1), lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    x, y, s = bf(4, 8), bf(4, 8), bf(4, 8)
    bad = [
        lambda: F.ftp_dropout(x, y, 0.5, None), lambda: F.ftp_dropout(x, y.float(), 0.5, words), lambda: F.ftp_dropout(x, bf(4, 9), 0.5, words),
        lambda: F.ftp_dropout(x, y, 0.5, words.int()), lambda: F.ftp_dropout(x, y, 0.5, words.cpu()), lambda: F.ftp_dropout(x.cpu(), y, 0.5, words),
        lambda: F.ftp_dropout(x, y, 1.5, words), lambda: F.ftp_dropout(x.half(), y.half(), 0.5, words), lambda: F.ftp_dropout(x.t(), y, 0.5, words),
        lambda: F.ftp_dropout(x, y, 0.5, words, site=-1),
        lambda: F.ftp_join_forward(x, y, s), lambda: F.ftp_join_forward(None, None, None, y), lambda: F.ftp_join_forward(x, y, None, s),
        lambda: F.ftp_join_forward(x, y, s, bf(3, 8)), lambda: F.ftp_join_forward(x, y, s, bf(4, 8), w_pre=bf(8)), lambda: F.ftp_join_forward(x, y, s, bf(4, 8), w_pre=f32(7)),
        lambda: F.ftp_join_forward(x, y, s, bf(4, 8), gate=bf(2, 8), gate_rows=3, stats=f32(4, 3)), lambda: F.ftp_join_forward(x, y, s, bf(4, 8), gate=bf(2, 8), gate_rows=1),
        lambda: F.ftp_join_forward(x, y, s, bf(4, 8), gate=bf(8)), lambda: F.ftp_join_forward(x, y, s, bf(4, 8), gate_rows=2), lambda: F.ftp_join_forward(x, y, s, bf(4, 8), dropout=0.1),
        lambda: F.ftp_join_forward(bf(1, 16400), bf(1, 16400), bf(1, 16400), bf(1, 16400)), lambda: F.ftp_join_forward(x, y, x, s),
        lambda: F.ftp_join_backward(x, y, s, None, None, du=bf(4, 8)), lambda: F.ftp_join_backward(x, y, None, None, f32(4, 4), du=bf(4, 8)),
        lambda: F.ftp_join_backward(x, y, s, None, f32(4, 4), du=bf(4, 8), dgate=f32(8)), lambda: F.ftp_join_backward(None, y, s, None, f32(4, 4), du=bf(4, 8)),
        lambda: F.ftp_join_backward(bf(400, 8), bf(400, 8), bf(400, 8), None, f32(4, 400), du=bf(400, 8), ws=f32(8)),
        lambda: F.ftp_recurrence_forward(x, y, s.float()), lambda: F.ftp_recurrence_forward(x, y, bf(4, 9)), lambda: F.ftp_recurrence_forward(x, y, s, h0=f32(7)),
        lambda: F.ftp_recurrence_forward(x, y, s, h1=bf(8)), lambda: F.ftp_recurrence_forward(x, y, s, states=f32(0, 8)), lambda: F.ftp_recurrence_forward(x, y, x),
        lambda: F.ftp_recurrence_forward(x, y, s, offsets=torch.zeros(3, dtype=torch.int64, device="cuda")), lambda: F.ftp_recurrence_forward(x[0], y[0], s[0]),
        lambda: F.ftp_recurrence_forward(bf(2, 2, 8), bf(2, 2, 8), bf(2, 2, 8), offsets=i32(3)), lambda: F.ftp_recurrence_forward(bf(8, 4).t(), y, s),
        lambda: F.ftp_recurrence_forward(bf(3, 4, 8)[:, :2], bf(3, 2, 8), bf(3, 2, 8)),          # a larger gap between sequences than between steps
        lambda: F.ftp_recurrence_backward(x, y, s, f32(1, 8), bf(4, 8), bf(4, 8), o=bf(4, 8)),
        lambda: F.ftp_logprob_forward(x, i32(3), f32(4)), lambda: F.ftp_logprob_forward(x, i32(4).long(), f32(4)), lambda: F.ftp_logprob_forward(x, None, f32(4)),
        lambda: F.ftp_logprob_forward(x, i32(4), f32(4), top=i32(4, 9)), lambda: F.ftp_logprob_forward(x, i32(4), f32(4), top_logp=f32(4, 2)),
        lambda: F.ftp_logprob_forward(x, i32(4), f32(4), lse=f32(4)), lambda: F.ftp_logprob_forward(x, i32(4), f32(4), scale=0.0),
        lambda: F.ftp_logprob_backward(x, i32(4), f32(4, 2), f32(4), bf(4, 7)), lambda: F.ftp_logprob_backward(x, i32(4), f32(4, 2), None, bf(4, 8)),
        lambda: F.ftp_logprob_backward(x, i32(4), f32(4, 2), f32(4), bf(4, 8), dentropy=f32(4)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((F.FtpError, AttributeError)):
            call()
            pytest.fail(str(i))
