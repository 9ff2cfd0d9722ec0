"""Operators around the feed-forward products on the GPU, where values or layouts are at their limits: states updated in place
across a cluster, tails of runs, the float range's ends, what lies under a dropped element, gates far from 0."""
import math
import subprocess
import sys
from pathlib import Path

import pytest
import torch

import token_helpers as H
from ffn_helpers import HALF, Guarded, assert_within
from test_gpu_token import BF, FP, close, gen, join_case, on_gpu, rec_inputs, rnd, rng_of, vec

F = pytest.importorskip("paper_2110_02781_b200")
pytestmark = pytest.mark.gpu


# ---- recurrence: one tensor for the states in front and behind --------------------------------------------------------
@pytest.mark.parametrize("seqs,steps,cols", [(1, 2048, 64), (1, 1000, 128), (2, 600, 96), (1, 2047, 31), (3, 700, 65)])
@pytest.mark.parametrize("dt", [BF, FP])
def test_states_in_place_of_one_another_in_one_turn_of_a_cluster(seqs, steps, cols, dt):
    g = gen("place", seqs, steps, cols)
    rows = seqs * steps
    f, v, o, dy = (rnd(g, seqs, steps, cols).to(dt).cuda() for _ in range(4))
    h0, dh1 = rnd(g, seqs, cols).float().cuda(), rnd(g, seqs, cols).float().cuda()
    states = torch.empty(F.ftp_recurrence_states(rows, seqs), cols, device="cuda")
    y, y2, h1 = torch.empty_like(f), torch.empty_like(f), torch.empty_like(h0)
    F.ftp_recurrence_forward(f, v, y, o=o, h0=h0, h1=h1, states=states)
    grads = [torch.empty_like(f) for _ in range(6)]
    dh0 = torch.empty_like(h0)
    F.ftp_recurrence_backward(f, v, dy, states, grads[0], grads[1], o=o, do=grads[2], dh1=dh1, dh0=dh0)
    for _ in range(20):
        h, dh = h0.clone(), dh1.clone()
        F.ftp_recurrence_forward(f, v, y2, o=o, h0=h, h1=h)
        F.ftp_recurrence_backward(f, v, dy, states, grads[3], grads[4], o=o, do=grads[5], dh1=dh, dh0=dh)
        assert torch.equal(y, y2) and torch.equal(h, h1) and torch.equal(dh, dh0)
        assert all(torch.equal(a, b) for a, b in zip(grads[:3], grads[3:]))


# ---- recurrence: tails of runs -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("seqs,steps,cols", [(300, 391, 64), (320, 200, 32), (150, 1003, 128)])
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("coupled", [True, False])
def test_backward_without_a_gate_walks_on_from_a_tail(seqs, steps, cols, dt, coupled):
    """Enough sequences that a block walks one alone, in several turns of which the first has a partial run."""
    g = gen("tail", seqs, steps, cols)
    rows = seqs * steps
    f, f64, v, v64, _, _ = rec_inputs(g, rows, cols, dt, coupled=coupled)
    dy, dy64 = on_gpu(rnd(g, rows, cols), dt)
    three = lambda t: t.view(seqs, steps, cols)  # noqa: E731
    y, df, dv = (torch.full((rows, cols), -7.0, dtype=dt, device="cuda") for _ in range(3))
    states = torch.empty(F.ftp_recurrence_states(rows, seqs), cols, device="cuda")
    how = dict(coupled=coupled, act=F.ACT_NONE)
    plain = lambda t: three(t.t.contiguous())  # noqa: E731
    F.ftp_recurrence_forward(plain(f), plain(v), three(y), states=states, **how)
    F.ftp_recurrence_backward(plain(f), plain(v), plain(dy), states, three(df), three(dv), **how)
    zero = torch.zeros(cols, dtype=torch.float64)
    for b in (0, seqs // 2, seqs - 1):
        at = slice(b * steps, (b + 1) * steps)
        want = H.recurrence_backward(f64[at], v64[at], None, zero, dy64[at], zero, None, coupled, dt)
        close(df[at], want["df"], dt, f"df of {b}")
        close(dv[at], want["dv"], dt, f"dv of {b}")


# ---- log probabilities: the float range's ends ---------------------------------------------------------------------------
def logprob_both_ways(x, t, scale, dt):
    """Forward with entropy, and the gradients of all three ways in, against 64 bits."""
    xd, x64 = x.to(dt).cuda(), x.to(dt).double()
    rows = x.shape[0]
    logp, ent, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
    F.ftp_logprob_forward(xd, t.cuda(), logp, entropy=ent, lse=lse, scale=scale)
    r_logp, r_ent, r_lse, _, e1, e2 = H.logprob(x64, t, scale)
    fin = torch.isfinite(r_logp.float())                                 # what a float can hold
    assert bool((logp.cpu()[~fin] == -math.inf).all())
    assert_within(logp.cpu()[fin], r_logp[fin], e1[fin], "logp")
    assert_within(ent, r_ent, e2, "entropy")
    assert torch.equal(lse[:, 0].double().cpu(), r_lse[:, 0])
    g = gen("ends", rows, x.shape[1])
    dl, dl64 = vec(rnd(g, rows))
    dh, dh64 = vec(rnd(g, rows))
    for a, b in ((dl, None), (None, dh), (dl, dh)):
        d = torch.empty_like(xd)
        F.ftp_logprob_backward(xd, t.cuda(), lse, a, d, entropy=ent, dentropy=b, scale=scale)
        close(d, H.logprob_backward(x64, t, scale, dl64 if a is not None else None, dh64 if b is not None else None), dt, "dlogits")


def rows_at_the_top(rows, vocab, dt):
    low, high = torch.finfo(dt).min, torch.finfo(dt).max
    x = torch.zeros(6, vocab, dtype=torch.float64)
    x[0, vocab // 2] = high                                              # a token that is forced
    x[1, 1] = x[1, vocab - 1] = high                                     # two of them
    x[2] = -math.inf
    x[2, vocab // 2], x[2, 3] = high, low                                # the whole range in one row
    x[3, vocab // 2] = 2.0e38
    x[4, vocab // 2], x[4, 2] = 2.5e38, 1.0e38
    x[5] = high                                                          # uniform
    return x[torch.arange(rows) % 6]


@pytest.mark.parametrize("rows,vocab", [(6, 40), (6, 9000), (6, 70000), (600, 40), (606, 9000), (3, 70000)])
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("scale", [1.0, 0.5, 1.5, 1000.0])
def test_logprob_of_logits_at_the_top_of_the_range(rows, vocab, dt, scale):
    t = torch.full((rows,), vocab // 2, dtype=torch.int32)
    t[1::2] = 1
    x = rows_at_the_top(rows, vocab, dt)
    logp, ent, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
    F.ftp_logprob_forward(x.to(dt).cuda(), t.cuda(), logp, entropy=ent, lse=lse, scale=scale)
    r_logp, r_ent, r_lse, _, e1, e2 = H.logprob(x.to(dt).double(), t, scale)
    fin = torch.isfinite(r_logp.float())                                 # what a float can hold
    assert bool((logp.cpu()[~fin] == -math.inf).all())
    assert_within(logp.cpu()[fin], r_logp[fin], e1[fin], "logp")
    assert_within(ent, r_ent, e2, "entropy")
    assert torch.equal(lse[:, 0].double().cpu(), r_lse[:, 0])


@pytest.mark.parametrize("rows,vocab", [(6, 40), (6, 9000), (606, 1001)])
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("scale", [1.0, 0.5, 1.5, 1000.0])
def test_logprob_gradients_at_the_top_of_the_range(rows, vocab, dt, scale):
    t = torch.full((rows,), vocab // 2, dtype=torch.int32)
    t[1::2] = 1
    logprob_both_ways(rows_at_the_top(rows, vocab, dt), t, scale, dt)


@pytest.mark.parametrize("rows,vocab", [(5, 40), (7, 9001), (600, 300)])
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("scale", [1e9, 1e12, 1e18])
def test_logprob_of_masked_rows_with_a_large_scale(rows, vocab, dt, scale):
    scale = float(torch.tensor(scale, dtype=torch.float32))
    x = rnd(gen("scale", rows, vocab), rows, vocab, scale=2.0) / scale
    x[:, 1::3] = -math.inf
    x[:, 2::5] = torch.finfo(dt).min
    logprob_both_ways(x, torch.zeros(rows, dtype=torch.int32), scale, dt)


# ---- joins: what lies under a dropped element ------------------------------------------------------------------------------
UNDER = [dict(post="none", pre="none", gate="vector"), dict(post="none", pre="rms", gate=None), dict(post="none", pre="layer", gate=7), dict(post="none", pre="rms", gate=1),
         dict(post="rms", pre="rms", gate="vector"), dict(post="layer", pre="layer", gate=1, bias=1), dict(post="rms", pre="none", gate=50), dict(post="layer", pre="rms", gate=None, bare=1)]


@pytest.mark.parametrize("rows,cols", [(40, 64), (67, 133), (30, 520), (12, 4096), (11, 2560), (9, 8192), (5, 9000), (4, 9001)])
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("how", UNDER, ids=lambda h: f"{h['post']}-{h['pre']}-{h['gate']}")
def test_whatever_lies_under_a_dropped_element_of_a_join(rows, cols, dt, how):
    g, own, ref = join_case(rows, cols, 0, 0, dt, {"p": 0.25, **how})
    own.pop("b_pre")
    gone = ref["mask"] == 0
    spoil = gone & (torch.rand(rows, cols, generator=g) < 0.2)
    bad = torch.where(torch.rand(rows, cols, generator=g) < 0.5, math.nan, math.inf).double()
    holes = lambda t: torch.where(spoil, bad, t)  # noqa: E731
    u, u64 = on_gpu(rnd(g, rows, cols), dt)
    s, s64 = on_gpu(rnd(g, rows, cols), dt)
    ds, ds64 = on_gpu(rnd(g, rows, cols), dt)
    dy, dy64 = on_gpu(rnd(g, rows, cols), dt)
    stats = torch.zeros(4, rows, dtype=torch.float64)
    for i, (kind, of) in enumerate(((how["post"], u64), (how["pre"], s64))):
        if kind != "none":
            mean, r = H.moments(of, kind, ref["eps"])
            stats[2 * i], stats[2 * i + 1] = mean[:, 0], r[:, 0]
    if how["post"] == "none":
        u.t.copy_(holes(u64).to(dt))
        out = torch.empty_like(u.t)
        F.ftp_join_forward(u.t, s.t, out, None, **{**own, "pre": F.NORM_NONE, "w_pre": None})
        close(out, H.join_forward(u64, s64, ref), dt, "s")
    ds.t.copy_(holes(ds64).to(dt))
    grads = {"d" + n: torch.empty(cols, device="cuda") for n in ("w_post", "b_post", "w_pre", "b_pre") if (how["post"] if "post" in n else how["pre"]) != "none"}
    if own["gate"] is not None:
        grads["dgate"] = torch.empty_like(own["gate"])
    du, dx = torch.empty_like(u.t), torch.empty_like(u.t)
    pre = how["pre"] != "none"
    F.ftp_join_backward(u.t, s.t if pre else None, dy.t if pre else None, ds.t, stats.float().cuda(), du=du, dx=dx, **grads, **own)
    want = H.join_backward(u64, s64, dy64, ds64, ref)
    for name, t in {**grads, "du": du}.items():
        close(t, want[name], t.dtype, name)
    assert not torch.isfinite(dx.cpu()[spoil]).any()                     # the stream's gradient passes on what came in
    dx.copy_(torch.where(spoil.cuda(), want["dx"][0].cuda(), dx.double()).to(dt))
    close(dx, want["dx"], dt, "dx")


# ---- recurrence: gates far from 0 ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("steps,cols", [(1, 64), (17, 33), (40, 64)])
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("far", [20.0, 40.0, 75.0])
def test_recurrence_gates_far_from_zero(steps, cols, dt, far):
    """a next to 0 and 1 - a next to 0, each relative to itself: the exponential (float: 2 units in the last place, 4 roundings; bf16: 2^-22 and a rounding of
    the exponent, |f| roundings of the value), an addition, a reciprocal and a product, then at most 8 more products."""
    g = gen("far", steps, cols, far)
    f64 = (far * (1.0 + torch.linspace(0, 0.05, cols, dtype=torch.float64))).expand(steps, cols).to(dt).double().clone()
    rel = (16 * H.U if dt == FP else 2.0 ** -21 + far * 1.05 * H.U + 12 * H.U)
    sign = torch.where(torch.arange(steps) % 2 == 0, 1.0, -1.0).double()[:, None]
    one = (1.0 + torch.rand(1, cols, generator=g, dtype=torch.float64)).to(dt).double()
    gpu = lambda t, d=dt: t.to(d).cuda()  # noqa: E731
    states = torch.empty(F.ftp_recurrence_states(steps, 1), cols, device="cuda")
    y, df, dv = (torch.empty(steps, cols, dtype=dt, device="cuda") for _ in range(3))
    h1, dh0 = torch.empty(1, cols, device="cuda"), torch.empty(1, cols, device="cuda")

    def both_ways(f, v, h0, dy, dh1):
        F.ftp_recurrence_forward(gpu(f), gpu(v), y, h0=gpu(h0, FP), h1=h1, states=states)
        F.ftp_recurrence_backward(gpu(f), gpu(v), gpu(dy), states, df, dv, dh1=gpu(dh1, FP), dh0=dh0)
    near = lambda got, want, what: assert_within(got, want, (rel + HALF[got.dtype]) * want.abs(), what)  # noqa: E731
    nothing = torch.zeros(steps, cols, dtype=torch.float64)
    # 1 - a: a first value that nothing adds to and nothing forgets (a is 1), and a gradient that reaches every step
    a, b = H.gates(f64)
    v = nothing.clone()
    v[0] = one
    both_ways(f64, v, nothing[:1], nothing, one)
    near(y, (b[0] * one).expand(steps, cols), "y")
    near(h1, b[:1] * one, "h1")
    near(dv, b * one, "dv")
    # a: every state is the step's own value, of the other sign than the last
    a, b = H.gates(-f64)
    v = sign * one
    both_ways(-f64, v, -v[:1], one.expand(steps, cols), nothing[:1])
    near(y, v, "y")
    near(df, a * b * one * (-2 * v), "df")
    near(dh0, a[:1] * one, "dh0")


def test_recurrence_output_gates_closed_by_the_lowest_value():
    """silu(o) and its slope are 0 far below 0: what reaches the states does not come through such an output."""
    for dt in (BF, FP):
        for cols in (64, 65):
            g = gen("closed", cols, str(dt))
            f, v, dy = (rnd(g, 50, cols).to(dt).cuda() for _ in range(3))
            dh1 = rnd(g, 1, cols).float().cuda()
            states = torch.empty(F.ftp_recurrence_states(50, 1), cols, device="cuda")
            res = []
            for value in (0.0, torch.finfo(dt).min, -1e35, -1e30, -200.0):
                o = torch.full_like(f, value)
                y, df, dv, do, dh0 = (*(torch.empty_like(f) for _ in range(4)), torch.empty_like(dh1))
                F.ftp_recurrence_forward(f, v, y, o=o, states=states)
                F.ftp_recurrence_backward(f, v, dy, states, df, dv, o=o, do=do, dh1=dh1, dh0=dh0)
                assert not y.float().abs().max() > 1e-30
                if value:
                    assert do.float().abs().max() < 1e-30
                res.append((df.float(), dv.float(), dh0))
            for other in res[1:]:
                for a, b in zip(res[0], other):
                    assert torch.allclose(a, b, rtol=1e-6, atol=1e-30)


def test_recurrence_packed_sequences_of_no_rows():
    for max_len in (None, 0, 40, 1000):
        e = lambda: torch.empty(0, 8, dtype=BF, device="cuda")  # noqa: E731
        off = torch.zeros(4, dtype=torch.int32, device="cuda")
        h0, h1 = torch.randn(3, 8, device="cuda"), torch.empty(3, 8, device="cuda")
        states = torch.full((F.ftp_recurrence_states(0, 3), 8), -7.0, device="cuda")
        F.ftp_recurrence_forward(e(), e(), e(), h0=h0, h1=h1, states=states, offsets=off, max_len=max_len)
        assert torch.equal(h0, h1) and bool((states == -7.0).all())
        F.ftp_recurrence_backward(e(), e(), e(), states, e(), e(), dh1=h0, dh0=h1.zero_(), offsets=off, max_len=max_len)
        assert torch.equal(h0, h1)


# ---- a launch that the runtime refuses -------------------------------------------------------------------------------------
def test_a_refused_launch_is_reported_once():
    """A launch into the legacy stream while a blocking stream of this thread is captured is an error of the host; the next call, outside the capture, is a
    call like any other."""
    code = """
import ctypes as C
import torch, paper_2110_02781_b200 as F
f32 = lambda *s: torch.randn(*s, device="cuda")
x, y, t, lp = f32(64, 256), f32(64, 256), torch.zeros(64, dtype=torch.int32, device="cuda"), f32(64)
f, v, h = f32(1, 300, 64), f32(1, 300, 64), f32(1, 300, 64)
calls = [lambda **k: F.ftp_logprob_forward(x, t, lp, **k), lambda **k: F.ftp_recurrence_forward(f, v, h, **k), lambda **k: F.ftp_dropout(x, y, 0.0, None, **k),
         lambda **k: F.ftp_join_forward(None, x, None, y, post=F.NORM_NONE, **k)]
for c in calls:
    c()
torch.cuda.synchronize()
cu = C.CDLL("libcuda.so.1")
def ok(r):
    assert r == 0, r
for bad in calls:
    st, graph = C.c_void_p(), C.c_void_p()
    ok(cu.cuStreamCreate(C.byref(st), 0))
    ok(cu.cuStreamBeginCapture_v2(st, 0))
    try:
        bad(stream=0)
        refused = False
    except F.FtpError as e:
        refused = "launch failed" in str(e)
    cu.cuStreamEndCapture(st, C.byref(graph))
    ok(cu.cuStreamDestroy_v2(st))
    assert refused
    for c in calls:
        c()
torch.cuda.synchronize()
print("reported once")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=str(Path(__file__).parent.parent))
    assert r.returncode == 0 and "reported once" in r.stdout, r.stdout + r.stderr


# ---- recurrence: columns of a wider tensor -----------------------------------------------------------------------------------
@pytest.mark.parametrize("cols,gap", [(63, 1), (7, 1), (1, 7), (33, 7), (66, 6), (130, 6), (61, 3), (5, 3)])
@pytest.mark.parametrize("lengths", [[700], [33] * 20, [64, 0, 5, 257, 16, 1], [100] * 300])
@pytest.mark.parametrize("dt,name", [(BF, "silu"), (BF, None), (FP, "silu"), (FP, None)])
def test_recurrence_over_rows_on_16_bytes_of_columns_that_are_not(cols, gap, lengths, dt, name):
    """Rows of every tensor start on 16 bytes, and the last columns do not fill theirs: what lies behind them is another's."""
    g = gen("slices", cols, str(lengths), name)
    rows, seqs = sum(lengths), len(lengths)
    f, f64, v, v64, o, o64 = rec_inputs(g, rows, cols, dt, gap)
    dy, dy64 = on_gpu(rnd(g, rows, cols), dt, gap)
    starts = [0] + torch.tensor(lengths).cumsum(0).tolist()
    y, df, dv, do = (Guarded(rows, cols, dt, gap) for _ in range(4))
    states = torch.empty(F.ftp_recurrence_states(rows, seqs), cols, device="cuda")
    how = dict(act=F.ACT_SILU if name else F.ACT_NONE, offsets=torch.tensor(starts, dtype=torch.int32, device="cuda"), max_len=max(lengths), o=o.t if name else None)
    F.ftp_recurrence_forward(f.t, v.t, y.t, states=states, **how)
    F.ftp_recurrence_backward(f.t, v.t, dy.t, states, df.t, dv.t, do=do.t if name else None, **how)
    assert y.untouched() and df.untouched() and dv.untouched() and do.untouched()
    zero = torch.zeros(cols, dtype=torch.float64)
    for b in sorted({0, seqs // 2, seqs - 1}):
        at = slice(starts[b], starts[b + 1])
        o1 = o64[at] if name else None
        _, _, ys, ey = H.recurrence(f64[at], v64[at], o1, zero, name, True, dt)
        want = H.recurrence_backward(f64[at], v64[at], o1, zero, dy64[at], zero, name, True, dt)
        close(y.t[at], (ys, ey), dt, f"y of {b}")
        close(df.t[at], want["df"], dt, f"df of {b}")
        close(dv.t[at], want["dv"], dt, f"dv of {b}")
        if name:
            close(do.t[at], want["do"], dt, f"do of {b}")


# ---- tensors of more than 2^31 elements ---------------------------------------------------------------------------------------
def test_wide_offsets_through_the_copy_engine_and_backward():
    """Rows whose elements lie beyond 2^31: long sequences, and the backward passes."""
    rows, cols, ld = 45, 96, 50_000_000
    buf = torch.zeros((rows - 1) * ld + 16 * cols, dtype=BF, device="cuda")
    far = [torch.as_strided(buf, (rows, cols), (ld, 1), i * cols) for i in range(12)]
    near = [torch.randn(rows, cols, device="cuda").to(BF) for _ in range(12)]
    for a, b in zip(far, near):
        a.copy_(b)

    def run(t):
        f, v, o, dy, y, df, dv, do, dl, du, dx, dg = t
        states, h1, dh0 = torch.empty(F.ftp_recurrence_states(rows, 1), cols, device="cuda"), torch.empty(1, cols, device="cuda"), torch.empty(1, cols, device="cuda")
        F.ftp_recurrence_forward(f, v, y, o=o, h1=h1, states=states)
        F.ftp_recurrence_backward(f, v, dy, states, df, dv, o=o, do=do, dh0=dh0)
        lse, lp = torch.empty(rows, 2, device="cuda"), torch.empty(rows, device="cuda")
        token = torch.arange(rows, dtype=torch.int32, device="cuda")
        F.ftp_logprob_forward(f, token, lp, lse=lse)
        F.ftp_logprob_backward(f, token, lse, lp, dl)
        stats, w, dw = torch.rand(4, rows, device="cuda", generator=torch.Generator("cuda").manual_seed(1)), torch.ones(cols, device="cuda"), torch.empty(2, cols, device="cuda")
        F.ftp_join_backward(f, v, o, dy, stats, du=du, dx=dx, dgate=dg, dw_post=dw[0], dw_pre=dw[1], gate=y, gate_rows=1, w_post=w, w_pre=w, dropout=0.2, rng=rng_of(3, 4))
        return [y, df, dv, do, dl, du, dx, dg, h1, dh0, lse, dw]
    for a, b in zip(run(far), run(near)):
        assert torch.equal(a, b)
