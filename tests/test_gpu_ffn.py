"""Feed-forward operators (linear, gated, 8-bit activation checkpoints) on the GPU against their float64 forms."""
import math
import os
import subprocess
import sys
import threading

import pytest
import torch

from ffn_helpers import (ACT_EVAL, ACT_SLOPE, ACTS, HALF, Guarded, act, assert_within, dact, product_err, through_8_bits)

pytestmark = pytest.mark.gpu
F = pytest.importorskip("paper_2110_02781_b200")
BF, FP = torch.bfloat16, torch.float32


def rnd(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g, dtype=torch.float64) * scale


def dev(x, dt, gap=0, off=0):
    """x on the GPU in dt, optionally as a view with gaps between rows, starting off elements into a buffer."""
    rows, cols = x.shape
    buf = torch.full((off + max(rows, 1) * (cols + gap),), math.nan, dtype=dt, device="cuda")
    v = buf[off:].view(max(rows, 1), cols + gap)[:rows, :cols]
    v.copy_(x.to(dt))
    return v


def ref(t):
    return t.double().cpu()


# ---- 8-bit images --------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,cols,gap,off", [(1, 1, 0, 0), (1, 31, 0, 0), (3, 32, 0, 0), (5, 33, 3, 1), (7, 100, 0, 0), (64, 256, 8, 0), (129, 1283, 0, 0), (2, 4096, 0, 8)])
@pytest.mark.parametrize("dt", [BF, FP])
def test_checkpoint_values_are_exact(rows, cols, gap, off, dt):
    x = rnd(1, rows, cols) * torch.exp2(rnd(2, rows, cols).mul(6).round())        # blocks of very different size
    x[0, : min(cols, 32)] = 0.0
    xd = dev(x, dt, gap, off)
    img = torch.full((F.ftp_checkpoint_bytes(rows, cols),), 0x5A, dtype=torch.uint8, device="cuda")
    F.ftp_checkpoint_pack(xd, img)
    out = Guarded(rows, cols, dt, gap, off)
    F.ftp_checkpoint_unpack(img, out.t)
    torch.cuda.synchronize()
    assert torch.equal(ref(out.t), through_8_bits(ref(xd)))                       # integers times powers of two: no tolerance
    assert out.untouched()
    err = (ref(out.t) - ref(xd)).abs()
    top = torch.stack([ref(xd)[:, a:a + 32].abs().amax(1) for a in range(0, cols, 32)], 1).repeat_interleave(32, 1)[:, :cols]
    assert (err <= top / 64 + 2.0 ** -127).all()                                  # one step where the largest code is cut to 127, half a step else
    other = torch.empty(rows, cols, dtype=FP if dt == BF else BF, device="cuda")  # the values fit either type
    F.ftp_checkpoint_unpack(img, other)
    assert torch.equal(ref(other), ref(out.t))


def test_checkpoint_extremes():
    big = torch.finfo(FP).max
    rows = [[big, -big, 1.0] + [0.0] * 29, [2.0 ** -149, -2.0 ** -140, 0.0] + [0.0] * 29, [2.0 ** -120] * 16 + [2.0 ** -127] * 16,
            [127.9, 127.4, 64.0, 0.5, -0.5, 1.5, 2.5, -127.9] + [0.0] * 24, [math.nan] + [1.0] * 31, [math.inf, -1.0] + [0.0] * 30]
    x = torch.tensor(rows, dtype=FP)
    img = torch.empty(F.ftp_checkpoint_bytes(6, 32), dtype=torch.uint8, device="cuda")
    out = torch.empty(6, 32, dtype=FP, device="cuda")
    F.ftp_checkpoint_pack(x.cuda(), img)
    F.ftp_checkpoint_unpack(img, out)
    want = through_8_bits(x.double())
    got = ref(out)
    assert torch.equal(got[:4], want[:4])
    assert torch.isnan(got[4:]).all() and torch.isnan(want[4:]).all()


def test_checkpoint_parts_do_not_touch_each_other():
    rows, cols = 37, 70
    xs = [dev(rnd(s, rows, cols), BF) for s in (3, 4, 5)]
    img = torch.empty(F.ftp_checkpoint_bytes(rows, cols, 3), dtype=torch.uint8, device="cuda")
    for i in (1, 0, 2):
        F.ftp_checkpoint_pack(xs[i], img, part=i)
    out = torch.empty(rows, cols, dtype=BF, device="cuda")
    for i in range(3):
        F.ftp_checkpoint_unpack(img, out, part=i)
        assert torch.equal(ref(out), through_8_bits(ref(xs[i])))


# ---- linear -----------------------------------------------------------------------------------------------
LINEAR = [  # rows, cin, cout, gap, off
    (1, 64, 64, 0, 0), (1, 1, 1, 0, 0), (1, 513, 77, 0, 0), (2, 200, 136, 0, 0), (3, 1000, 40, 8, 0), (8, 256, 512, 0, 0), (9, 72, 24, 0, 0),
    (16, 2048, 128, 0, 0), (31, 33, 35, 1, 1), (128, 128, 128, 0, 0), (129, 65, 129, 0, 8), (200, 1283, 517, 0, 0), (257, 320, 1280, 0, 0),
    (300, 8, 1000, 4, 2), (513, 777, 264, 0, 0)]

# a few tokens: long and short reductions, strips of columns that end early, rows of w on odd addresses
FEW = [(1, 4096, 256, 0, 0), (2, 1024, 70, 0, 0), (4, 520, 129, 0, 1), (5, 2000, 33, 8, 0), (7, 31, 300, 3, 0), (1, 30000, 40, 0, 0), (8, 9000, 72, 0, 0),
       (13, 600, 100, 0, 0), (16, 1025, 36, 0, 1), (17, 300, 65, 0, 0), (29, 2100, 40, 4, 0), (32, 64, 33, 0, 0), (30, 9000, 24, 0, 0), (1, 2000, 72, 0, 0),
       (2, 640, 64, 8, 8), (3, 1300, 200, 0, 0), (4, 130, 1000, 0, 0), (6, 2048, 104, 0, 0), (47, 500, 68, 0, 0), (48, 72, 260, 0, 0), (49, 72, 260, 0, 0)]
# enough output tiles for CTA pairs: forward, input gradient, weight gradient; odd edges, several tiles per pair
LARGE = [(1000, 330, 2300, 0, 0), (1100, 72, 2104, 8, 0), (3001, 40, 2300, 0, 0), (1000, 2300, 330, 0, 0), (330, 1000, 2300, 0, 0), (70, 1100, 2104, 0, 8),
         (1023, 2049, 33, 0, 0), (2305, 64, 1025, 0, 0)]
# the same with results, addends and kept values whose rows lie on 2, 4 or 8 bytes
UNEVEN = [(2500, 300, 2051, 0, 0), (2500, 300, 2050, 0, 0), (1300, 500, 2053, 1, 2), (2500, 2051, 300, 0, 0), (2500, 2050, 300, 0, 1), (1400, 2060, 300, 0, 0)]


# few output tiles over a long reduction: clusters of CTA pairs that share tiles, in the forward pass or a gradient
SHARED = [(130, 1283, 2050, 0, 0), (300, 4100, 1100, 0, 0), (300, 1100, 4100, 8, 0), (130, 1100, 4100, 0, 0), (2050, 4100, 200, 0, 8), (2050, 200, 4100, 0, 0),
          (1290, 200, 2050, 0, 0)]


def linear_case(seed, rows, cin, cout, dt, gap, off):
    x, w = dev(rnd(seed, rows, cin), dt, gap, off), dev(rnd(seed + 1, cin, cout, scale=cin ** -0.5), dt, gap, off)
    return x, w


@pytest.mark.parametrize("rows,cin,cout,gap,off", LINEAR + FEW + LARGE + UNEVEN + SHARED + [(1100, 8000, 2051, 0, 0), (1100, 8000, 2050, 0, 0)])
@pytest.mark.parametrize("dt,name,bias,res,keep", [(BF, "gelu", 1, 1, "full"), (BF, "none", 0, 0, None), (FP, "silu", 1, 1, "8bit"), (FP, "relu6", 0, 1, "full"),
                                                   (BF, "silu", 1, 0, None), (FP, "gelu", 1, 1, None), (BF, "relu", 0, 1, "8bit")])
def test_linear_forward(rows, cin, cout, gap, off, dt, name, bias, res, keep):
    x, w = linear_case(10, rows, cin, cout, dt, gap, off)
    b = rnd(12, cout).float().cuda() if bias else None
    r = dev(rnd(13, rows, cout), dt, gap, off) if res else None
    y = Guarded(rows, cout, dt, gap, off)
    stash = None
    if keep == "full":
        stash = torch.full((rows, cout), math.nan, dtype=dt, device="cuda")
    elif keep == "8bit":
        stash = torch.zeros(F.ftp_checkpoint_bytes(rows, cout), dtype=torch.uint8, device="cuda")
    F.ftp_linear_forward(x, w, y.t, bias=b, residual=r, act=ACTS[name], stash=stash)
    F.ftp_check_op_status()
    z = ref(x) @ ref(w) + (ref(b) if bias else 0.0)
    ez = product_err(ref(x).abs() @ ref(w).abs(), cin, dt) + 2.0 ** -23 * z.abs()
    a = act(z, name)
    want = a + (ref(r) if res else 0.0)
    bound = ACT_SLOPE * ez + (ACT_EVAL * z.abs().clamp(min=1) if name in ("gelu", "silu") else 0.0) + 2.0 ** -23 * (a.abs() + want.abs())
    assert_within(y.t, want, bound + HALF[dt] * (want.abs() + bound), "y")
    assert y.untouched()
    if keep == "full":
        assert_within(stash, z, ez + HALF[dt] * (z.abs() + ez), "stash")
    elif keep == "8bit":
        out = torch.empty(rows, cout, dtype=FP, device="cuda")
        F.ftp_checkpoint_unpack(stash, out)
        top = torch.stack([(z.abs() + ez)[:, c:c + 32].amax(1) for c in range(0, cout, 32)], 1).repeat_interleave(32, 1)[:, :cout]
        assert_within(out, z, ez + top / 64, "stash")


@pytest.mark.parametrize("rows,cin,cout,gap,off", [c for c in LINEAR if c[0] != 16] + [(1100, 40, 56, 0, 0), (5000, 16, 16, 0, 0)] + LARGE + UNEVEN + SHARED)
@pytest.mark.parametrize("dt,name,x8,keep,wide", [(BF, "gelu", 0, "full", 0), (BF, "none", 0, None, 1), (FP, "silu", 0, "full", 0), (FP, "none", 1, None, 0),
                                                  (BF, "relu6", 1, "8bit", 1), (FP, "gelu", 1, "8bit", 0)])
def test_linear_backward(rows, cin, cout, gap, off, dt, name, x8, keep, wide):
    x, w = linear_case(20, rows, cin, cout, dt, gap, off)
    dy = dev(rnd(22, rows, cout), dt, gap, off)
    add = dev(rnd(23, rows, cin), dt, gap, off)
    zd = dev(rnd(24, rows, cout, scale=2.0), dt)
    stash, z = None, None
    if keep == "full":
        stash, z = zd, ref(zd)
    elif keep == "8bit":
        stash, z = torch.empty(F.ftp_checkpoint_bytes(rows, cout), dtype=torch.uint8, device="cuda"), through_8_bits(ref(zd))
        F.ftp_checkpoint_pack(zd, stash)
    xin, xv = x, ref(x)
    if x8:
        xin, xv = torch.empty(F.ftp_checkpoint_bytes(rows, cin), dtype=torch.uint8, device="cuda"), through_8_bits(xv)
        F.ftp_checkpoint_pack(x, xin)
    dtw = FP if wide else dt
    dx, dw, db = Guarded(rows, cin, dt, gap, off), Guarded(cin, cout, dtw, gap, off), torch.full((cout,), math.nan, device="cuda")
    F.ftp_linear_backward(xin, w, dy, dx=dx.t, dw=dw.t, dbias=db, act=ACTS[name], stash=stash, dx_addend=add)
    F.ftp_check_op_status()
    dz = ref(dy) * (dact(z, name) if z is not None else 1.0)
    smooth = name in ("gelu", "silu")
    e0 = ref(dy).abs() * ACT_EVAL * z.abs().clamp(min=1) if smooth else torch.zeros_like(dz)
    # bf16: dz is rounded before the products (unless dy passes unchanged)
    e1 = e0 + ((HALF[BF] * (dz.abs() + e0)) if dt == BF and z is not None else 2.0 ** -23 * dz.abs())
    want = dz @ ref(w).T + ref(add)
    bound = e1 @ ref(w).abs().T + product_err((dz.abs() + e1) @ ref(w).abs().T, cout, dt) + 2.0 ** -23 * want.abs()
    assert_within(dx.t, want, bound + HALF[dt] * (want.abs() + bound), "dx")
    want = xv.T @ dz
    bound = xv.abs().T @ e1 + product_err(xv.abs().T @ (dz.abs() + e1), rows, dt)
    assert_within(dw.t, want, bound + HALF[dtw] * (want.abs() + bound), "dw")
    want = dz.sum(0)
    # 64 rows or fewer per float sum, then double
    assert_within(db, want, e0.sum(0) + 2.0 ** -23 * 24 * (dz.abs() + e0).sum(0), "dbias")
    assert dx.untouched() and dw.untouched()


# ---- gated --------------------------------------------------------------------------------------------------
GATED = [(1, 64, 64, 0, 0), (1, 1, 1, 0, 0), (1, 1000, 333, 0, 0), (4, 130, 200, 0, 0), (8, 512, 96, 8, 0), (33, 100, 31, 1, 1), (128, 256, 128, 0, 0),
         (130, 72, 136, 0, 0), (257, 1283, 320, 0, 0), (300, 64, 1000, 0, 8), (1000, 330, 1150, 0, 0), (1100, 72, 1048, 8, 0), (70, 1100, 1052, 0, 0),
         (1025, 2049, 33, 0, 0), (130, 4100, 700, 0, 0), (130, 1283, 1100, 0, 0), (300, 1100, 2050, 8, 0), (130, 1100, 1100, 0, 0), (2050, 700, 200, 0, 8)]


def kept_pair(keep, rows, cout, dt, seed):
    """(stash tensor, its two planes in float64) for a backward pass."""
    gu = torch.stack([rnd(seed, rows, cout, scale=2.0), rnd(seed + 1, rows, cout)]).to(dt).cuda()
    if keep == "full":
        return gu, ref(gu)
    img = torch.empty(F.ftp_checkpoint_bytes(rows, cout, 2), dtype=torch.uint8, device="cuda")
    for i in range(2):
        F.ftp_checkpoint_pack(gu[i], img, part=i)
    return img, torch.stack([through_8_bits(ref(gu[i])) for i in range(2)])


@pytest.mark.parametrize("rows,cin,cout,gap,off", GATED + FEW)
@pytest.mark.parametrize("dt,name,keep", [(BF, "silu", None), (BF, "gelu", "full"), (FP, "silu", "8bit"), (FP, "none", None), (BF, "relu", "8bit"), (FP, "gelu", "full")])
def test_gated_forward(rows, cin, cout, gap, off, dt, name, keep):
    x, wg = linear_case(30, rows, cin, cout, dt, gap, off)
    _, wu = linear_case(40, rows, cin, cout, dt, gap, off)
    h = Guarded(rows, cout, dt, gap, off)
    stash = None
    if keep == "full":
        stash = torch.full((2, rows, cout), math.nan, dtype=dt, device="cuda")
    elif keep == "8bit":
        stash = torch.zeros(F.ftp_checkpoint_bytes(rows, cout, 2), dtype=torch.uint8, device="cuda")
    F.ftp_gated_forward(x, wg, wu, h.t, act=ACTS[name], stash=stash)
    F.ftp_check_op_status()
    g, u = ref(x) @ ref(wg), ref(x) @ ref(wu)
    eg, eu = (product_err(ref(x).abs() @ ref(w).abs(), cin, dt) for w in (wg, wu))
    a = act(g, name)
    ea = ACT_SLOPE * eg + (ACT_EVAL * g.abs().clamp(min=1) if name in ("gelu", "silu") else 0.0)
    want = a * u
    bound = ea * (u.abs() + eu) + a.abs() * eu + 2.0 ** -23 * want.abs()
    assert_within(h.t, want, bound + HALF[dt] * (want.abs() + bound), "h")
    assert h.untouched()
    for i, (v, e) in enumerate(((g, eg), (u, eu))):
        if keep == "full":
            assert_within(stash[i], v, e + HALF[dt] * (v.abs() + e), f"stash[{i}]")
        elif keep == "8bit":
            out = torch.empty(rows, cout, dtype=FP, device="cuda")
            F.ftp_checkpoint_unpack(stash, out, part=i)
            top = torch.stack([(v.abs() + e)[:, c:c + 32].amax(1) for c in range(0, cout, 32)], 1).repeat_interleave(32, 1)[:, :cout]
            assert_within(out, v, e + top / 64, f"stash[{i}]")


def gated_bounds(x, wg, wu, g, u, dh, name, dt, eg=0.0, eu=0.0):
    """dg, du and the bounds of what enters the products, from the kept values (eg, eu: how far those may be off)."""
    a, da = act(g, name), dact(g, name)
    ev = ACT_EVAL * g.abs().clamp(min=1) if name in ("gelu", "silu") else torch.zeros_like(g)
    ea, eda = ev + ACT_SLOPE * eg, ev + ACT_SLOPE * eg
    dg, du = dh * u * da, dh * a
    e_g = dh.abs() * (u.abs() * eda + eu * (da.abs() + eda)) + 2.0 ** -22 * dg.abs()
    e_u = dh.abs() * ea + 2.0 ** -23 * du.abs()
    if dt == BF:
        e_g, e_u = e_g + HALF[BF] * (dg.abs() + e_g), e_u + HALF[BF] * (du.abs() + e_u)
    return dg, du, e_g, e_u


def check_gated_grads(x, wg, wu, dg, du, e_g, e_u, add, dx, dws, dt, dtw, rows, cout):
    want = dg @ wg.T + du @ wu.T + add
    mag = (dg.abs() + e_g) @ wg.abs().T + (du.abs() + e_u) @ wu.abs().T
    bound = e_g @ wg.abs().T + e_u @ wu.abs().T + product_err(mag, 2 * cout + 64, dt) + 2.0 ** -23 * want.abs()
    assert_within(dx, want, bound + HALF[dt] * (want.abs() + bound), "dx")
    for d, e, t, n in ((dg, e_g, dws[0], "dw_gate"), (du, e_u, dws[1], "dw_up")):
        want = x.T @ d
        bound = x.abs().T @ e + product_err(x.abs().T @ (d.abs() + e), rows, dt)
        assert_within(t, want, bound + HALF[dtw] * (want.abs() + bound), n)


@pytest.mark.parametrize("rows,cin,cout,gap,off", GATED + [(1500, 24, 40, 0, 0)])
@pytest.mark.parametrize("dt,name,x8,keep,wide", [(BF, "silu", 0, "full", 0), (BF, "gelu", 1, "8bit", 1), (FP, "silu", 0, "8bit", 0), (FP, "gelu", 1, "full", 0),
                                                  (FP, "relu6", 0, "full", 0), (BF, "none", 0, "8bit", 0)])
def test_gated_backward(rows, cin, cout, gap, off, dt, name, x8, keep, wide):
    x, wg = linear_case(50, rows, cin, cout, dt, gap, off)
    _, wu = linear_case(60, rows, cin, cout, dt, gap, off)
    dh, add = dev(rnd(70, rows, cout), dt, gap, off), dev(rnd(71, rows, cin), dt, gap, off)
    stash, (g, u) = kept_pair(keep, rows, cout, dt, 72)
    xin, xv = x, ref(x)
    if x8:
        xin, xv = torch.empty(F.ftp_checkpoint_bytes(rows, cin), dtype=torch.uint8, device="cuda"), through_8_bits(xv)
        F.ftp_checkpoint_pack(x, xin)
    dtw = FP if wide else dt
    dx, dwg, dwu = Guarded(rows, cin, dt, gap, off), Guarded(cin, cout, dtw, gap, off), Guarded(cin, cout, dtw, gap, off)
    F.ftp_gated_backward(xin, wg, wu, dh, dx=dx.t, dw_gate=dwg.t, dw_up=dwu.t, act=ACTS[name], stash=stash, dx_addend=add)
    F.ftp_check_op_status()
    dg, du, e_g, e_u = gated_bounds(xv, ref(wg), ref(wu), g, u, ref(dh), name, dt)
    check_gated_grads(xv, ref(wg), ref(wu), dg, du, e_g, e_u, ref(add), dx.t, (dwg.t, dwu.t), dt, dtw, rows, cout)
    assert dx.untouched() and dwg.untouched() and dwu.untouched()


@pytest.mark.parametrize("dt,x8", [(BF, 0), (FP, 0), (BF, 1), (FP, 1)])
def test_gated_backward_computes_the_products_again(dt, x8):
    rows, cin, cout, name = 150, 96, 200, "silu"
    x, wg = linear_case(80, rows, cin, cout, dt, 0, 0)
    _, wu = linear_case(90, rows, cin, cout, dt, 0, 0)
    dh = dev(rnd(95, rows, cout), dt)
    xin, xv = x, ref(x)
    if x8:
        xin, xv = torch.empty(F.ftp_checkpoint_bytes(rows, cin), dtype=torch.uint8, device="cuda"), through_8_bits(xv)
        F.ftp_checkpoint_pack(x, xin)
    dx, dwg, dwu = (torch.empty(*s, dtype=dt, device="cuda") for s in ((rows, cin), (cin, cout), (cin, cout)))
    F.ftp_gated_backward(xin, wg, wu, dh, dx=dx, dw_gate=dwg, dw_up=dwu, act=ACTS[name])
    F.ftp_check_op_status()
    g, u = xv @ ref(wg), xv @ ref(wu)
    eg, eu = (product_err(xv.abs() @ ref(w).abs(), cin, dt) for w in (wg, wu))
    eg, eu = eg + HALF[dt] * (g.abs() + eg), eu + HALF[dt] * (u.abs() + eu)       # they are kept in the tensors' type
    dg, du, e_g, e_u = gated_bounds(xv, ref(wg), ref(wu), g, u, ref(dh), name, dt, eg, eu)
    check_gated_grads(xv, ref(wg), ref(wu), dg, du, e_g, e_u, 0.0, dx, (dwg, dwu), dt, dt, rows, cout)


# ---- gradients against differences of the forward pass -------------------------------------------------------
@pytest.mark.parametrize("name", ["none", "gelu", "silu"])
def test_linear_gradients_match_differences(name):
    rows, cin, cout, h = 9, 21, 17, 2.0 ** -8
    x, w = dev(rnd(100, rows, cin), FP), dev(rnd(101, cin, cout, scale=0.3), FP)
    b, dy = rnd(102, cout).float().cuda(), dev(rnd(103, rows, cout), FP)
    y, z = torch.empty(rows, cout, device="cuda"), torch.empty(rows, cout, device="cuda")
    stash = None if name == "none" else z

    def loss(xx, ww, bb):
        F.ftp_linear_forward(xx, ww, y, bias=bb, act=ACTS[name])
        return float((ref(y) * ref(dy)).sum())
    F.ftp_linear_forward(x, w, y, bias=b, act=ACTS[name], stash=stash)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    F.ftp_linear_backward(x, w, dy, dx=dx, dw=dw, dbias=db, act=ACTS[name], stash=stash)
    # central differences: the third derivative of an activation is below 2, so a term's cut-off error is below
    # |dy| |v|^3 h^2 / 3; rounding: 2^-20 of the terms summed, over 2 h
    g = torch.Generator().manual_seed(7)
    for t, grad, pos in ((x, dx, 0), (w, dw, 1), (b, db, 2)):
        v = torch.randn(t.shape, generator=g).cuda()
        args = [x, w, b]
        args[pos] = t + h * v
        up = loss(*args)
        args[pos] = t - h * v
        down = loss(*args)
        dzv = ref(v) @ ref(w) if pos == 0 else ref(x) @ ref(v) if pos == 1 else ref(v).expand(rows, cout)
        cut = float((ref(dy).abs() * dzv.abs() ** 3).sum()) * h * h / 3
        noise = float((ref(dy).abs() * (ref(x).abs() @ ref(w).abs() + ref(b).abs() + 1)).sum()) * 2.0 ** -20 / (2 * h)
        assert abs((up - down) / (2 * h) - float((ref(grad) * ref(v)).sum())) <= cut + 2 * noise + 1e-6, pos


# ---- masks, non-finite values, sharing ------------------------------------------------------------------------
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("rows", [3, 140])
def test_non_finite_rows_stay_in_their_row(dt, rows):
    cin, cout = 200, 72
    x = rnd(110, rows, cin)
    x[1, 5], x[rows - 1, 7] = math.nan, math.inf
    xd, w = dev(x, dt), dev(rnd(111, cin, cout), dt)
    y, clean = torch.empty(rows, cout, dtype=dt, device="cuda"), torch.empty(rows, cout, dtype=dt, device="cuda")
    h = torch.empty(rows, cout, dtype=dt, device="cuda")
    F.ftp_linear_forward(xd, w, y, act=F.ACT_SILU)
    F.ftp_gated_forward(xd, w, w, h)
    xz = x.clone()
    xz[1], xz[rows - 1] = 0.0, 0.0
    F.ftp_linear_forward(dev(xz, dt), w, clean, act=F.ACT_SILU)
    keep = [r for r in range(rows) if r not in (1, rows - 1)]
    assert torch.equal(y[keep], clean[keep]) and torch.isfinite(h[keep]).all()
    assert torch.isnan(y[1]).all() and torch.isnan(h[1]).all() and not torch.isfinite(ref(h[rows - 1])).all()
    assert (clean[1] == 0).all()


@pytest.mark.parametrize("name", list(ACTS))
def test_extreme_values_before_the_activation(name):
    # z = x w with w the identity: what the activation and its derivative do with zeros, huge values and NaN
    v = torch.tensor([[0.0, -0.0, 1e-30, -1e-30, 50.0, -50.0, 1e4, -1e4, 3e38, -3e38, 6.0, -6.0, 5.999, 100.0, -100.0, -20.0]])
    eye = torch.eye(16)
    for dt in (BF, FP):
        z = dev(v.expand(130, 16).double(), dt)
        y = torch.empty(130, 16, dtype=dt, device="cuda")
        F.ftp_linear_forward(z, dev(eye.double(), dt), y, act=ACTS[name])
        want = act(ref(z), name)
        assert_within(y, want, (HALF[dt] + ACT_EVAL) * want.abs() + ACT_EVAL * 2.0 ** -2, "y")
        ones, dx = torch.ones(130, 16, dtype=dt, device="cuda"), torch.empty(130, 16, dtype=dt, device="cuda")
        F.ftp_linear_backward(None, dev(eye.double(), dt), ones, dx=dx, act=ACTS[name], stash=None if name == "none" else z.contiguous())
        want = dact(ref(z), name)
        assert_within(dx, want, 2 * HALF[dt] * want.abs() + ACT_EVAL * 2.0 ** 3, "dx")


def test_residual_may_be_the_output_and_addend_may_be_dx():
    rows, cin, cout = 130, 72, 200
    x, w = linear_case(120, rows, cin, cout, BF, 0, 0)
    r = dev(rnd(121, rows, cout), BF)
    y, inplace = torch.empty_like(r), r.clone()
    F.ftp_linear_forward(x, w, y, residual=r, act=F.ACT_GELU)
    F.ftp_linear_forward(x, w, inplace, residual=inplace, act=F.ACT_GELU)
    assert torch.equal(y, inplace)
    a = dev(rnd(122, rows, cin), BF)
    dx, inplace = torch.empty_like(a), a.clone()
    F.ftp_linear_backward(None, w, y, dx=dx, dx_addend=a)
    F.ftp_linear_backward(None, w, y, dx=inplace, dx_addend=inplace)
    assert torch.equal(dx, inplace)


def test_weights_may_be_halves_of_one_matrix():
    rows, cin, f = 70, 136, 96
    both = dev(rnd(130, cin, 2 * f), BF)
    x, dh = dev(rnd(131, rows, cin), BF), dev(rnd(132, rows, f), BF)
    outs = []
    for wg, wu in ((both[:, :f], both[:, f:]), (both[:, :f].contiguous(), both[:, f:].contiguous())):
        h, stash = torch.empty(rows, f, dtype=BF, device="cuda"), torch.empty(2, rows, f, dtype=BF, device="cuda")
        F.ftp_gated_forward(x, wg, wu, h, stash=stash)
        d = torch.empty(cin, 2 * f, dtype=BF, device="cuda")
        dx = torch.empty_like(x)
        F.ftp_gated_backward(x, wg, wu, dh, dx=dx, dw_gate=d[:, :f], dw_up=d[:, f:], stash=stash)
        outs.append((h, stash, d, dx))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_no_rows():
    w = dev(rnd(140, 40, 24), BF)
    empty = lambda c: torch.empty(0, c, dtype=BF, device="cuda")  # noqa: E731
    F.ftp_linear_forward(empty(40), w, empty(24), residual=empty(24))
    F.ftp_gated_forward(empty(40), w, w, empty(24))
    dw, dw2, db = (torch.full(s, 5.0, dtype=t, device="cuda") for s, t in (((40, 24), BF), ((40, 24), BF), ((24,), FP)))
    F.ftp_linear_backward(empty(40), w, empty(24), dx=empty(40), dw=dw, dbias=db)
    assert (dw == 0).all() and (db == 0).all()
    dw.fill_(5.0)
    F.ftp_gated_backward(empty(40), w, w, empty(24), dx=empty(40), dw_gate=dw, dw_up=dw2)
    assert (dw == 0).all() and (dw2 == 0).all()
    F.ftp_checkpoint_pack(empty(40), torch.empty(0, dtype=torch.uint8, device="cuda"))
    F.ftp_check_op_status()


# ---- as they are used together ----------------------------------------------------------------------------------
def block_step(x, wg, wu, wd, dy, bufs):
    """One training step of y = (act(x wg) * (x wu)) wd + x that keeps everything in 8 bits."""
    rows, d, f = x.shape[0], x.shape[1], wg.shape[1]
    F.ftp_checkpoint_pack(x, bufs["x8"])
    F.ftp_gated_forward(x, wg, wu, bufs["h"], stash=bufs["pre8"])
    F.ftp_checkpoint_pack(bufs["h"], bufs["h8"])
    F.ftp_linear_forward(bufs["h"], wd, bufs["y"], residual=x)
    F.ftp_linear_backward(bufs["h8"], wd, dy, dx=bufs["dh"], dw=bufs["dwd"])
    F.ftp_gated_backward(bufs["x8"], wg, wu, bufs["dh"], dx=bufs["dx"], dw_gate=bufs["dwg"], dw_up=bufs["dwu"], stash=bufs["pre8"], dx_addend=dy)


def block_buffers(rows, d, f, dt):
    e = lambda *s: torch.full(s, math.nan, dtype=dt, device="cuda")  # noqa: E731
    i = lambda *a: torch.empty(F.ftp_checkpoint_bytes(*a), dtype=torch.uint8, device="cuda")  # noqa: E731
    return dict(x8=i(rows, d), pre8=i(rows, f, 2), h8=i(rows, f), h=e(rows, f), y=e(rows, d), dh=e(rows, f), dx=e(rows, d), dwg=e(d, f), dwu=e(d, f), dwd=e(f, d))


@pytest.mark.parametrize("rows,d,f", [(1, 64, 128), (130, 96, 264), (300, 100, 130)])
def test_block_step_from_8_bit_checkpoints(rows, d, f):
    dt = BF
    x, wg = linear_case(150, rows, d, f, dt, 0, 0)
    _, wu = linear_case(160, rows, d, f, dt, 0, 0)
    wd, dy = dev(rnd(170, f, d, scale=f ** -0.5), dt), dev(rnd(171, rows, d), dt)
    b = block_buffers(rows, d, f, dt)
    block_step(x, wg, wu, wd, dy, b)
    F.ftp_check_op_status()
    # every operator against its own inputs as the GPU has them: what one hands to the next is exact
    h, dh = ref(b["h"]), ref(b["dh"])
    want = h @ ref(wd) + ref(x)
    e = product_err(h.abs() @ ref(wd).abs(), f, dt) + 2.0 ** -23 * want.abs()
    assert_within(b["y"], want, e + HALF[dt] * (want.abs() + e), "y")
    want = ref(dy) @ ref(wd).T
    e = product_err(ref(dy).abs() @ ref(wd).abs().T, d, dt)
    assert_within(b["dh"], want, e + HALF[dt] * (want.abs() + e), "dh")
    h8 = through_8_bits(h)
    want = h8.T @ ref(dy)
    e = product_err(h8.abs().T @ ref(dy).abs(), rows, dt)
    assert_within(b["dwd"], want, e + HALF[dt] * (want.abs() + e), "dwd")
    gu = torch.empty(2, rows, f, device="cuda")
    for i in range(2):
        F.ftp_checkpoint_unpack(b["pre8"], gu[i], part=i)
    x8 = through_8_bits(ref(x))
    dg, du, e_g, e_u = gated_bounds(x8, ref(wg), ref(wu), ref(gu[0]), ref(gu[1]), dh, "silu", dt)
    check_gated_grads(x8, ref(wg), ref(wu), dg, du, e_g, e_u, ref(dy), b["dx"], (b["dwg"], b["dwu"]), dt, dt, rows, f)


def test_captured_step_replays_with_new_inputs_and_matches_eager_calls():
    rows, d, f, dt = 140, 72, 200, BF
    mk = lambda s: [dev(rnd(s + i, *shape, scale=sc), dt) for i, (shape, sc) in enumerate((((rows, d), 1.0), ((d, f), 0.1), ((d, f), 0.1), ((f, d), 0.1), ((rows, d), 1.0)))]  # noqa: E731
    live, other = mk(180), mk(190)
    b = block_buffers(rows, d, f, dt)
    eager = block_buffers(rows, d, f, dt)
    block_step(*live, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block_step(*live, b)
    for a, o in zip(live, other):
        a.copy_(o)
    graph.replay()
    block_step(*other, eager)
    torch.cuda.synchronize()
    for k in b:
        if b[k].dtype == dt:
            assert torch.equal(b[k], eager[k]), k
    F.ftp_check_op_status()


def test_calls_on_another_stream_and_on_two_streams_at_once():
    rows, cin, cout = 600, 264, 520
    x, w = linear_case(200, rows, cin, cout, FP, 0, 0)
    z, dy = dev(rnd(202, rows, cout), FP), dev(rnd(203, rows, cout), FP)

    def grads(stream):
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(cout, device="cuda")
        F.ftp_linear_backward(x, w, dy, dx=dx, dw=dw, dbias=db, act=F.ACT_GELU, stash=z, stream=stream)
        return dx, dw, db
    want = grads(None)
    torch.cuda.synchronize()
    ss = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [grads(ss[i % 2]) for i in range(6)]
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))            # and the same bits every time


def test_wide_offsets():
    # a view whose rows lie far apart: element offsets beyond 2^31
    rows, cin, cout, ld = 3, 64, 48, (1 << 30) + 8
    big = torch.empty(2 * ld + cin, dtype=BF, device="cuda")
    x = torch.as_strided(big, (rows, cin), (ld, 1))
    x.copy_(rnd(210, rows, cin).to(BF))
    w = dev(rnd(211, cin, cout), BF)
    y, y2 = torch.empty(rows, cout, dtype=BF, device="cuda"), torch.empty(rows, cout, dtype=BF, device="cuda")
    F.ftp_linear_forward(x, w, y, act=F.ACT_SILU)
    F.ftp_linear_forward(x.contiguous(), w, y2, act=F.ACT_SILU)
    assert torch.equal(y, y2)
    img = torch.empty(F.ftp_checkpoint_bytes(rows, cin), dtype=torch.uint8, device="cuda")
    F.ftp_checkpoint_pack(x, img)
    out = torch.empty(rows, cin, dtype=BF, device="cuda")
    F.ftp_checkpoint_unpack(img, out)
    assert torch.equal(ref(out), through_8_bits(ref(x)))


# ---- refusals of the binding --------------------------------------------------------------------------------------
def test_refusals():
    x, w, y = dev(rnd(220, 10, 32), BF), dev(rnd(221, 32, 24), BF), torch.empty(10, 24, dtype=BF, device="cuda")
    bias, dw, db = torch.zeros(24, device="cuda"), torch.empty_like(w), torch.empty(24, device="cuda")
    img = lambda *a: torch.empty(F.ftp_checkpoint_bytes(*a), dtype=torch.uint8, device="cuda")  # noqa: E731
    r, both = torch.zeros_like(y), torch.zeros(2, 10, 24, dtype=BF, device="cuda")
    F.ftp_linear_forward(x, w, y, bias=bias)
    bad = [
        lambda: F.ftp_linear_forward(x.float(), w, y),                              # types differ
        lambda: F.ftp_linear_forward(x.cpu(), w, y),
        lambda: F.ftp_linear_forward(x.half(), w.half(), y.half()),
        lambda: F.ftp_linear_forward(x[:, :31], w, y),
        lambda: F.ftp_linear_forward(x, w, y[:9]),
        lambda: F.ftp_linear_forward(x, w, y.T.contiguous().T),                     # columns contiguous
        lambda: F.ftp_linear_forward(x[:1].expand(10, 32), w, y),                   # rows overlap
        lambda: F.ftp_linear_forward(x, w, y, bias=bias.to(BF)),
        lambda: F.ftp_linear_forward(x, w, y, bias=bias[:23]),
        lambda: F.ftp_linear_forward(x, w, y, residual=y[:5]),
        lambda: F.ftp_linear_forward(x, w, y, act=9),
        lambda: F.ftp_linear_forward(x, w, y, stash=torch.empty(10, 23, dtype=BF, device="cuda")),
        lambda: F.ftp_linear_forward(x, w, y, stash=img(9, 24)[:-1]),
        lambda: F.ftp_linear_backward(x, w, y, dw=dw, act=F.ACT_GELU),               # no kept values
        lambda: F.ftp_linear_backward(x, w, y, dw=dw, stash=torch.empty_like(y)),    # nothing to keep them for
        lambda: F.ftp_linear_backward(None, w, y, dw=dw),
        lambda: F.ftp_linear_backward(x, w, y, dw=dw[:31]),
        lambda: F.ftp_linear_backward(x, w, y, dw=dw, dx_addend=x),                  # nothing to add it to
        lambda: F.ftp_linear_backward(img(9, 32)[:64], w, y, dw=dw),
        lambda: F.ftp_linear_backward(x, w, y, dbias=db[:3]),
        lambda: F.ftp_gated_forward(x, w, w[:, :23], y),
        lambda: F.ftp_gated_forward(x, w, w),                                        # neither h nor kept values
        lambda: F.ftp_gated_backward(x, w, w, y, dw_gate=dw),
        lambda: F.ftp_gated_backward(None, w, w, y, dx=torch.empty_like(x)),         # products cannot be computed again
        lambda: F.ftp_linear_backward(x.float(), w.float(), y.float(), dw=dw.float(), ws=torch.empty(16, dtype=torch.uint8, device="cuda")),
        lambda: F.ftp_checkpoint_pack(x, img(9, 32)[:-300] if img(9, 32).numel() > 300 else img(1, 1)[:8]),
        lambda: F.ftp_checkpoint_pack(x.half(), img(10, 32)),
        lambda: F.ftp_checkpoint_pack(x[0, 0], img(10, 32)),
        lambda: F.ftp_linear_forward(x.new_empty(2, 5, 0), w[:0], y),
        lambda: F.ftp_linear_forward(x, w[:, :8], x[:, :8]),                          # outputs on inputs or on each other
        lambda: F.ftp_linear_forward(x, w, y, stash=y),
        lambda: F.ftp_linear_forward(x, w, y, residual=r, stash=r),
        lambda: F.ftp_linear_backward(x, w, y, dw=w),
        lambda: F.ftp_linear_backward(x, w, y, dx=x),
        lambda: F.ftp_linear_backward(x, w[:, :8], x[:, :8], dx=x),
        lambda: F.ftp_gated_forward(x, w, w, both[0], stash=both),
        lambda: F.ftp_gated_backward(x, w, w, y, dw_gate=dw, dw_up=dw),
        lambda: F.ftp_checkpoint_unpack(img(10, 32, 2)[1:-255], x),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(F.FtpError):
            call()
            pytest.fail(f"call {k} was not refused")
    F.ftp_check_op_status()


def test_status_check_is_refused_while_the_stream_is_captured():
    F.ftp_check_op_status()
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g.capture_begin()
        torch.zeros(1, device="cuda")
        with pytest.raises(F.FtpError) as e:
            F.ftp_check_op_status()
        g.capture_end()
    assert e.value.status == 5
    F.ftp_check_op_status()


def test_first_calls_of_a_process_may_be_captured():
    code = """
import sys, torch
import paper_2110_02781_b200 as F
torch.manual_seed(0)
for dt, rows in ((torch.bfloat16, 1), (torch.bfloat16, 300), (torch.float32, 700)):
    x, w = torch.randn(rows, 72, device='cuda').to(dt), torch.randn(72, 136, device='cuda').to(dt)
    y, h, dx, dw = (torch.empty(*s, dtype=dt, device='cuda') for s in ((rows, 136), (rows, 136), (rows, 72), (72, 136)))
    img = torch.empty(F.ftp_checkpoint_bytes(rows, 72), dtype=torch.uint8, device='cuda')
    def step():
        F.ftp_linear_forward(x, w, y)
        F.ftp_gated_forward(x, w, w, h)
        F.ftp_checkpoint_pack(x, img)
        F.ftp_linear_backward(img, w, h, dx=dx, dw=dw)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for t in (y, h, dx, dw):
        t.zero_()
    g.replay()
    got = [t.clone() for t in (y, h, dx, dw)]
    step()
    F.ftp_check_op_status()
    assert all(torch.equal(a, b) for a, b in zip(got, (y, h, dx, dw)))
"""
    done = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


def test_calls_from_several_threads_at_once():
    shapes = [(1, 640, 512), (300, 200, 136), (130, 1100, 1100), (777, 264, 517)]
    cases = [(dev(rnd(300 + i, m, k), dt), dev(rnd(310 + i, k, n, scale=k ** -0.5), dt)) for i, (m, k, n) in enumerate(shapes) for dt in (BF, FP)]
    dys = [dev(rnd(320 + i, x.shape[0], w.shape[1]), x.dtype) for i, (x, w) in enumerate(cases)]

    def step(i):
        x, w = cases[i]
        y, h, dx, dw = x.new_empty(x.shape[0], w.shape[1]), x.new_empty(x.shape[0], w.shape[1]), torch.empty_like(x), torch.empty_like(w)
        F.ftp_linear_forward(x, w, y, act=F.ACT_SILU)
        F.ftp_gated_forward(x, w, w, h)
        F.ftp_linear_backward(x, w, dys[i], dx=dx, dw=dw)
        return y, h, dx, dw

    want = [step(i) for i in range(len(cases))]
    torch.cuda.synchronize()
    got, failed = {}, []

    def work(t):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(5):
                    for i in range(t, len(cases), 4):
                        got[t, i] = step(i)
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=(t,)) for t in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    F.ftp_check_op_status()
    assert not failed, failed
    assert len(got) == len(cases) and all(torch.equal(a, b) for (t, i), r in got.items() for a, b in zip(r, want[i]))


def test_an_addend_in_place_keeps_gaps_and_refuses_another_pitch():
    rows, cin, cout = 130, 72, 200
    x, w = linear_case(400, rows, cin, cout, BF, 0, 0)
    r, a = rnd(401, rows, cout), rnd(402, rows, cin)
    y, inplace = torch.empty(rows, cout, dtype=BF, device="cuda"), Guarded(rows, cout, BF, 24, fill=r)
    F.ftp_linear_forward(x, w, y, residual=dev(r, BF), act=F.ACT_SILU)
    F.ftp_linear_forward(x, w, inplace.t, residual=inplace.t, act=F.ACT_SILU)
    dx, din = torch.empty(rows, cin, dtype=BF, device="cuda"), Guarded(rows, cin, BF, 16, fill=a)
    F.ftp_linear_backward(None, w, y, dx=dx, dx_addend=dev(a, BF))
    F.ftp_linear_backward(None, w, y, dx=din.t, dx_addend=din.t)
    assert torch.equal(y, inplace.t) and torch.equal(dx, din.t) and inplace.untouched() and din.untouched()
    wide = torch.zeros(2 * rows, cout, dtype=BF, device="cuda")
    every_other, packed = wide.view(rows, 2 * cout)[:, :cout], wide[:rows]           # the same first row, other rows elsewhere
    for res, out in ((every_other, packed), (packed, every_other)):
        with pytest.raises(F.FtpError):
            F.ftp_linear_forward(x, w, out, residual=res)
    wide = torch.zeros(2 * rows, cin, dtype=BF, device="cuda")
    with pytest.raises(F.FtpError):
        F.ftp_linear_backward(None, w, y, dx=wide[:rows], dx_addend=wide.view(rows, 2 * cin)[:, :cin])
    one = torch.zeros(1, cout, dtype=BF, device="cuda")
    F.ftp_linear_forward(x[:1], w, one, residual=torch.as_strided(one, (1, cout), (2 * cout, 1)))       # one row has no pitch
    F.ftp_check_op_status()


@pytest.mark.parametrize("rows,cin,cout,gap,off", [(1, 64, 64, 0, 0), (3, 130, 200, 0, 0), (9, 72, 24, 8, 0), (33, 100, 31, 1, 1), (300, 64, 1000, 0, 8), (1000, 330, 1150, 0, 0),
                                                   (130, 4100, 700, 0, 0)])
@pytest.mark.parametrize("dt,name,x8,wide", [(BF, "gelu", 0, 1), (BF, "none", 1, 0), (FP, "relu6", 0, 0), (FP, "gelu", 1, 0), (BF, "silu", 1, 1), (FP, "silu", 0, 0)])
def test_products_computed_again_over_shapes_and_activations(rows, cin, cout, gap, off, dt, name, x8, wide):
    x, wg = linear_case(410, rows, cin, cout, dt, gap, off)
    _, wu = linear_case(420, rows, cin, cout, dt, gap, off)
    dh, add = dev(rnd(430, rows, cout), dt, gap, off), dev(rnd(431, rows, cin), dt, gap, off)
    xin, xv = x, ref(x)
    if x8:
        xin, xv = torch.empty(F.ftp_checkpoint_bytes(rows, cin), dtype=torch.uint8, device="cuda"), through_8_bits(xv)
        F.ftp_checkpoint_pack(x, xin)
    dtw = FP if wide else dt
    dx, dwg, dwu = Guarded(rows, cin, dt, gap, off), Guarded(cin, cout, dtw, gap, off), Guarded(cin, cout, dtw, gap, off)
    F.ftp_gated_backward(xin, wg, wu, dh, dx=dx.t, dw_gate=dwg.t, dw_up=dwu.t, act=ACTS[name], dx_addend=add)
    F.ftp_check_op_status()
    g, u = xv @ ref(wg), xv @ ref(wu)
    eg, eu = (product_err(xv.abs() @ ref(w).abs(), cin, dt) for w in (wg, wu))
    eg, eu = eg + HALF[dt] * (g.abs() + eg), eu + HALF[dt] * (u.abs() + eu)       # kept in the tensors' type
    dg, du, e_g, e_u = gated_bounds(xv, ref(wg), ref(wu), g, u, ref(dh), name, dt, eg, eu)
    if name == "relu6":                                                             # a g that may lie on either side of a kink
        near = (g.abs() <= eg) | ((g - 6).abs() <= eg)
        e_g = e_g + torch.where(near, ref(dh).abs() * (u.abs() + eu), torch.zeros_like(u)) * (1 + HALF[dt])
    check_gated_grads(xv, ref(wg), ref(wu), dg, du, e_g, e_u, ref(add), dx.t, (dwg.t, dwu.t), dt, dtw, rows, cout)
    assert dx.untouched() and dwg.untouched() and dwu.untouched()
    only = Guarded(rows, cin, dt, gap, off)                                        # one gradient alone, laid out alike: the same bits
    F.ftp_gated_backward(xin, wg, wu, dh, dx=only.t, act=ACTS[name], dx_addend=add)
    assert torch.equal(only.t, dx.t) and only.untouched()
