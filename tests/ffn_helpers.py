"""Plain float64 forms of the feed-forward operators and the error bounds their kernels are held to.

Bounds are elementwise and come from the arithmetic: half a step per rounding to a tensor's type, and for a product of
length K one float rounding (2^-23, the accumulator may cut instead of round) per 16-element step of the tensor cores, of
which float tensors take six (their plane pairs), on the sum of the magnitudes; the plane pairs left out are below 2^-24."""
import math

import torch

ACTS = {"none": 0, "relu": 1, "relu6": 2, "gelu": 3, "silu": 4}
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def act(z, name):
    if name == "none":
        return z
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "relu6":
        return z.clamp(0, 6)
    if name == "silu":
        return z * torch.sigmoid(z)
    return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))


def dact(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).double()
    if name == "relu6":
        return ((z > 0) & (z < 6)).double()
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def product_err(absprod, k, dt):
    """Bound of a product's float accumulation, from the product of the magnitudes and its length."""
    steps = (6 if dt == torch.float32 else 1) * -(-k // 16) + 16          # + 16: the terms inside a step, the slices of the reduction
    return steps * 2.0 ** -23 * absprod


# |act'| and |act''| never exceed 1.2 (gelu: 1.13 and 0.8, silu: 1.1 and 0.5); evaluating an activation or its derivative
# in float costs at most 2^-18 of max(1, |z|): hardware exponential 2^-21 |z| relative on bf16 tensors, erf 2^-22
ACT_SLOPE, ACT_EVAL = 1.2, 2.0 ** -18


def assert_within(got, ref, bound, what):
    got = got.double().cpu()
    ref, bound = ref.double().cpu(), bound.double().cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.isfinite(got).all(), f"{what}: non-finite values"
    over = (got - ref).abs() - bound
    if over.numel():
        i = int(over.argmax())
        assert over.flatten()[i] <= 0, f"{what}: {got.flatten()[i]} for {ref.flatten()[i]}, bound {bound.flatten()[i]} at {i} ({int((over > 0).sum())} off)"


def through_8_bits(x):
    """Values of the 8-bit image of x (float64 in, float64 out), block by block."""
    rows, cols = x.shape
    out = torch.empty_like(x)
    for a in range(0, cols, 32):
        v = x[:, a:a + 32]
        top = v.abs().amax(1, keepdim=True)
        _, e = torch.frexp(top)                                           # top = m 2^e, 0.5 <= m < 1
        s = torch.ldexp(torch.ones_like(top), (e - 7).clamp(min=-126))
        s = torch.where(top == 0, torch.full_like(s, 2.0 ** -126), s)
        out[:, a:a + 32] = (v / s).round().clamp(-127, 127) * s
        out[:, a:a + 32] = torch.where(torch.isfinite(v).all(1, keepdim=True), out[:, a:a + 32], torch.full_like(v, math.nan))
    return out


class Guarded:
    """A rows x cols tensor inside a larger buffer filled with a pattern: written(…) tells whether anything around it changed."""

    def __init__(self, rows, cols, dt, gap=0, off=0, fill=None):
        self.buf = torch.full((64 + off + max(rows, 1) * (cols + gap) + 64,), -7.0, dtype=dt, device="cuda")
        self.t = self.buf[64 + off:64 + off + max(rows, 1) * (cols + gap)].view(max(rows, 1), cols + gap)[:rows, :cols]
        if fill is not None:
            self.t.copy_(fill)

    def untouched(self):
        b = self.buf.clone()
        n = self.t.shape
        if n[0]:
            torch.as_strided(b, n, (self.t.stride(0), 1), self.t.storage_offset()).fill_(-7.0)
        return bool((b == -7.0).all())
