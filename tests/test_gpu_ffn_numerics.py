"""Values of the feed-forward operators where an elementwise worst-case bound says nothing: infinities, the
far ends of the activations, errors in the norm, sums of one sign, long sums."""
import math

import pytest
import torch

from ffn_helpers import ACTS, act, dact, product_err

pytestmark = pytest.mark.gpu
F = pytest.importorskip("paper_2110_02781_b200")
BF, FP = torch.bfloat16, torch.float32


def rnd(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def positive(seed, *shape):
    return 0.5 + torch.rand(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def ref(t):
    return t.double().cpu()


def same_kinds(got, want):
    """The same NaN and the same infinities."""
    got, want = ref(got), ref(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf], want[inf])


# ---- infinities: products of a few tokens, of one CTA a tile, of clusters of pairs, of pairs -------------------------------
@pytest.mark.parametrize("rows,cin,cout", [(3, 200, 72), (20, 200, 72), (140, 200, 72), (140, 4100, 200), (1100, 72, 2104), (300, 4100, 1100)])
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("name", ["none", "relu6"])
def test_infinities_reach_the_results_that_hold_them(rows, cin, cout, dt, name):
    x, w = rnd(1, rows, cin), rnd(2, cin, cout)
    w[5, :8] = torch.tensor([1.0, -1.0, 0.0, 0.5, 3.0, -2.0, -0.0, 1.5])     # values of one plane, and zeros
    x[0, 5], x[1, 5] = math.inf, -math.inf
    x[2, 5], x[2, 9] = math.inf, math.inf                                    # of either sign in one sum
    w[7, 20], w[8, 21] = math.inf, -math.inf
    x[rows - 1, 7] = 1.0
    xd, wd = x.to(dt).cuda(), w.to(dt).cuda()
    y = torch.empty(rows, cout, dtype=dt, device="cuda")
    F.ftp_linear_forward(xd, wd, y, act=ACTS[name])
    same_kinds(y, act(ref(xd) @ ref(wd), name))


@pytest.mark.parametrize("rows,cin,cout", [(3, 200, 72), (12, 200, 72), (140, 200, 72), (1100, 72, 1052), (130, 4100, 700)])
@pytest.mark.parametrize("dt", [BF, FP])
def test_infinities_pass_through_the_gate(rows, cin, cout, dt):
    x, wg, wu = rnd(3, rows, cin), rnd(4, cin, cout), rnd(5, cin, cout)
    x[1, 5], x[rows - 1, 9] = math.inf, -math.inf
    xd, gd, ud = x.to(dt).cuda(), wg.to(dt).cuda(), wu.to(dt).cuda()
    h, kept = torch.empty(rows, cout, dtype=dt, device="cuda"), torch.empty(2, rows, cout, dtype=dt, device="cuda")
    F.ftp_gated_forward(xd, gd, ud, h, act=F.ACT_RELU, stash=kept)
    g, u = ref(xd) @ ref(gd), ref(xd) @ ref(ud)
    same_kinds(kept, torch.stack((g, u)))
    same_kinds(h, act(g, "relu") * u)


@pytest.mark.parametrize("rows,cin,cout", [(5, 200, 72), (140, 200, 72), (300, 1100, 900), (1100, 72, 2104)])
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("eight", [0, 1])
def test_infinities_pass_through_the_gradients(rows, cin, cout, dt, eight):
    x, w, dy = rnd(6, rows, cin), rnd(7, cin, cout), rnd(8, rows, cout)
    dy[2, 3], dy[4, 30] = math.inf, -math.inf
    xd, wd, dyd = x.to(dt).cuda(), w.to(dt).cuda(), dy.to(dt).cuda()
    xin, xv = xd, ref(xd)
    if eight:                                                                # one plane against three
        xin, back = torch.empty(F.ftp_checkpoint_bytes(rows, cin), dtype=torch.uint8, device="cuda"), torch.empty_like(xd)
        F.ftp_checkpoint_pack(xd, xin)
        F.ftp_checkpoint_unpack(xin, back)
        xv = ref(back)
    dx, dw = torch.empty_like(xd), torch.empty_like(wd)
    F.ftp_linear_backward(xin, wd, dyd, dx=dx, dw=dw)
    same_kinds(dx, ref(dyd) @ ref(wd).T)
    same_kinds(dw, xv.T @ ref(dyd))


# ---- GELU far from zero -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows", [3, 130])
def test_float_gelu_holds_its_accuracy_for_negative_values(rows):
    # z = x w with w the identity, exact.  Phi(z) = erfc(-z / sqrt 2) / 2: the argument is off by 2^-23 relative, which erfc turns
    # into (z^2 + 1) 2^-23 of its value, erfc itself by 4 steps and the product by one: (z^2 + 6) 2^-23 of the result.
    n = 64
    z = torch.linspace(-11.5, 9.0, rows * n, dtype=torch.float64).view(rows, n).float().cuda()
    eye = torch.eye(n, device="cuda")
    y, kept, dx = torch.empty_like(z), torch.empty_like(z), torch.empty_like(z)
    F.ftp_linear_forward(z, eye, y, act=F.ACT_GELU, stash=kept)
    assert torch.equal(kept, z)
    want = act(ref(z), "gelu")
    over = (ref(y) - want).abs() / ((ref(z) ** 2 + 6) * 2.0 ** -23 * want.abs()).clamp(min=2.0 ** -149)
    assert over.max() <= 1, (float(over.max()), float(ref(z).flatten()[over.argmax()]))
    # the derivative Phi + z phi: exp(-z^2 / 2) is off by (z^2 / 2 + 2) 2^-23 and both terms by two roundings, on the sum of the
    # magnitudes; its three planes hold it exactly
    F.ftp_linear_backward(None, eye, torch.ones_like(z), dx=dx, act=F.ACT_GELU, stash=kept)
    v = ref(z)
    size = 0.5 * torch.special.erfc(-v / math.sqrt(2)) + (v * torch.exp(-v * v / 2)).abs() / math.sqrt(2 * math.pi)
    over = (ref(dx) - dact(v, "gelu")).abs() / ((v ** 2 + 8) * 2.0 ** -23 * size)
    assert over.max() <= 1, (float(over.max()), float(v.flatten()[over.argmax()]))


# ---- errors in the norm -----------------------------------------------------------------------------------------------------
# A tile's accumulator takes 16 steps of 16 elements before it is added in float: every step cuts at most 2^-23, half of that on
# average, of a sum that grows to the chunk's, which makes 5e-7 of the result for terms of one sign and less for random ones;
# float additions of the chunks and the products left out (2^-24) add 2e-7.  Without the third plane it would be 3.5e-6, with
# the whole reduction in the accumulator 3e-5 for 1024 steps of one sign.
NORM = 1e-6


def off(got, want):
    return float((ref(got) - want).norm() / want.norm())


@pytest.mark.parametrize("rows,cin,cout", [(8, 9000, 72), (30, 9000, 24), (47, 5000, 68), (130, 16384, 140), (300, 4100, 1100), (1100, 4000, 2051), (200, 1283, 517),
                                           (2305, 2050, 1025)])
@pytest.mark.parametrize("make", [rnd, positive])
def test_float_products_keep_24_bits(rows, cin, cout, make):
    x, w, dy = make(11, rows, cin).float().cuda(), make(12, cin, cout).float().cuda(), make(13, rows, cout).float().cuda()
    y, h, kept = torch.empty(rows, cout, device="cuda"), torch.empty(rows, cout, device="cuda"), torch.empty(2, rows, cout, device="cuda")
    F.ftp_linear_forward(x, w, y)
    want = ref(x) @ ref(w)
    assert off(y, want) <= NORM
    w2 = make(14, cin, cout).float().cuda()
    F.ftp_gated_forward(x, w, w2, h, act=F.ACT_NONE, stash=kept)
    up = ref(x) @ ref(w2)
    assert off(kept[0], want) <= NORM and off(kept[1], up) <= NORM and off(h, want * up) <= 2 * NORM
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    F.ftp_linear_backward(x, w, dy, dx=dx, dw=dw)
    assert off(dx, ref(dy) @ ref(w).T) <= NORM and off(dw, ref(x).T @ ref(dy)) <= NORM


@pytest.mark.parametrize("rows,cin,cout", [(5000, 136, 200), (16384, 130, 70), (9000, 1032, 520)])
@pytest.mark.parametrize("make", [rnd, positive])
@pytest.mark.parametrize("dt,eight", [(FP, 0), (FP, 1), (BF, 0)])
def test_float_weight_gradients_of_long_batches(rows, cin, cout, make, dt, eight):
    x, dy = make(15, rows, cin).to(dt).cuda(), make(16, rows, cout).to(dt).cuda()
    w = torch.zeros(cin, cout, dtype=dt, device="cuda")
    xin, xv = x, ref(x)
    if eight:
        xin, back = torch.empty(F.ftp_checkpoint_bytes(rows, cin), dtype=torch.uint8, device="cuda"), torch.empty_like(x)
        F.ftp_checkpoint_pack(x, xin)
        F.ftp_checkpoint_unpack(xin, back)
        xv = ref(back)
    dw, db = torch.empty(cin, cout, device="cuda"), torch.empty(cout, device="cuda")
    F.ftp_linear_backward(xin, w, dy, dw=dw, dbias=db)
    assert off(dw, xv.T @ ref(dy)) <= NORM
    if make is positive:
        assert off(db, ref(dy).sum(0)) <= NORM


@pytest.mark.parametrize("rows", [8, 140, 1100])
@pytest.mark.parametrize("size", [-100, -115, -126, -135])
def test_float_operands_next_to_the_smallest_numbers(rows, size):
    # three planes end at bf16's smallest number, 2^-133: an operand is off by 2^-134 at most, times what it is multiplied with;
    # results below 2^-126 by half of 2^-149 more
    x, w = rnd(23, rows, 200).float(), rnd(24, 200, 300).float()
    y = torch.empty(rows, 300, device="cuda")
    for a, b in ((x * 2.0 ** size, w), (x, w * 2.0 ** size)):
        F.ftp_linear_forward(a.cuda(), b.cuda(), y)
        a, b = a.double(), b.double()
        bound = 2.0 ** -134 * (b.abs().sum(0) if a.abs().max() < b.abs().max() else a.abs().sum(1, keepdim=True)) + product_err(a.abs() @ b.abs(), 200, FP) + 2.0 ** -149
        over = (ref(y) - a @ b).abs() - bound
        assert over.max() <= 0, float(over.max())


# ---- long sums --------------------------------------------------------------------------------------------------------------
def test_bias_gradient_of_a_very_long_batch():
    # a column of one value each: rounding errors of a float sum do not cancel.  64 additions or fewer in float, the rest in double
    rows, cout = 1 << 23, 24
    c = positive(17, cout).float().cuda()
    dy = c.expand(rows, cout).contiguous()
    db = torch.empty(cout, device="cuda")
    F.ftp_linear_backward(None, torch.zeros(8, cout, device="cuda"), dy, dbias=db)
    err = (ref(db) / (rows * ref(c)) - 1).abs().max()
    assert err <= 68 * 2.0 ** -24, float(err)


def test_bf16_weight_gradient_of_a_very_long_batch():
    # terms of one sign: what the accumulator of the tensor cores cuts adds up.  Half a step of bf16 and 2^-14 for the sum
    rows, cin, cout = 1 << 23, 64, 72
    g = torch.Generator(device="cuda").manual_seed(18)
    make = lambda n: (0.5 + torch.rand(rows, n, generator=g, device="cuda")).to(BF)  # noqa: E731
    x, dy = make(cin), make(cout)
    dw = torch.empty(cin, cout, dtype=BF, device="cuda")
    F.ftp_linear_backward(x, torch.zeros(cin, cout, dtype=BF, device="cuda"), dy, dw=dw)
    want = sum(x[a:a + (1 << 20)].double().T @ dy[a:a + (1 << 20)].double() for a in range(0, rows, 1 << 20))
    err = ((dw.double() - want) / want).abs().max()
    assert err <= 2.0 ** -8 + 2.0 ** -14, float(err)


@pytest.mark.parametrize("rows,cin,cout", [(40, 1100000, 72), (300, 1100000, 392), (700, 300000, 1032), (700, 140000, 2304), (130, 70000, 72)])
def test_bf16_products_over_long_reductions(rows, cin, cout):
    # Sums too long for the accumulator, on one to four pairs a tile: forward, gated, input gradient (over cout), weight gradient
    # (over rows).  A chunk is 256 steps, which cut at most 2^-23 of its magnitudes each; 300 float additions at most: 2^-14.
    g = torch.Generator(device="cuda").manual_seed(19)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF)  # noqa: E731
    x, w, w2, res = make(rows, cin), make(cin, cout), make(cin, cout), make(rows, cout)
    new = lambda *s: torch.empty(*s, dtype=BF, device="cuda")  # noqa: E731

    def check(got, want, size, err=2.0 ** -14):
        over = (got.double() - want).abs() - (2.0 ** -8 + 2.0 ** -20) * want.abs() - err * size
        assert over.max() <= 0, float(over.max())
    xd = x.double()
    a, b, size = xd @ w.double(), xd @ w2.double(), xd.abs() @ torch.maximum(w.abs(), w2.abs()).double()
    y, h, kept = new(rows, cout), new(rows, cout), new(2, rows, cout)
    F.ftp_linear_forward(x, w, y, residual=res)
    check(y, a + res.double(), size)
    F.ftp_gated_forward(x, w, w2, h, act=F.ACT_NONE, stash=kept)
    check(kept[0], a, size)
    check(kept[1], b, size)
    check(h, a * b, size * (a.abs() + b.abs() + 2.0 ** -14 * size))
    # the same numbers as gradients: dx = dy w^T + addend, dw = x^T dy
    dx, dw = new(rows, cout), new(rows, cout)
    F.ftp_linear_backward(None, w.T.contiguous(), x, dx=dx, dx_addend=res)
    check(dx, a + res.double(), size)
    xt = x.T.contiguous()
    F.ftp_linear_backward(xt, res, w, dw=dw)
    check(dw, a, size)
    # dg = dh u and du = dh g with dh = g = w and u = w2: products of bf16 values, rounded to bf16 once more before the product
    grads = new(2, rows, cout)
    F.ftp_gated_backward(xt, res, res, w, dw_gate=grads[0], dw_up=grads[1], act=F.ACT_NONE, stash=torch.stack((w, w2)))
    for got, d in zip(grads, (w.double() * w2.double(), w.double() ** 2)):
        check(got, xd @ d.to(BF).double(), xd.abs() @ d.abs())
    F.ftp_check_op_status()
