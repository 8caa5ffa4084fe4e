"""Plain 64-bit forms of the layer-side operators, with bounds of what fp32 arithmetic may add to them.

A value is carried with a bound of its error: every fp32 operation adds at most U of its result, a sum of C values taken by 64 lanes and more
(at most 64 values in a lane, then a tree) at most (64 + 12) U of the sum of the magnitudes."""
import torch

U = 2.0 ** -24
SUM = 76 * U
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


# ---- rotary: the fraction of a revolution in fp32 is at most 2^-26 off (1.6 U radians), sine and cosine 2 units in the last place (4 U at 1); two
# products and a sum.  In 64 bits an angle of either side is rounded: here the product (2^-53 of it), in the kernel 2 pi, the quotient by it and
# the product (3 * 2^-53 together), so the sides differ by 2^-51 of the angle besides: 2 U at 2^29 radians, 30 U at 2^33
def rotary(x, pos, axis, freq, half):
    """x [T, H, D], pos [T, axes] -> (turned values, bound) in 64 bits."""
    x, P = x.double().cpu(), len(axis)
    angle = pos.double().cpu()[:, list(axis)] * torch.tensor(freq, dtype=torch.float64)
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    ia, ib = (slice(0, P), slice(P, 2 * P)) if half else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    out, bound = x.clone(), torch.zeros_like(x)
    a, b = x[..., ia], x[..., ib]
    out[..., ia], out[..., ib] = a * cos - b * sin, a * sin + b * cos
    bound[..., ia] = bound[..., ib] = (8 * U + 2.0 ** -51 * angle.abs()[:, None]) * (a.abs() + b.abs())
    return out, bound


# ---- norms
class Bounded:
    def __init__(self, v, e=0.0):
        self.v, self.e = v, torch.zeros_like(v) + e

    def times(self, w):
        v = self.v * w
        return Bounded(v, self.e * abs(w) + U * v.abs())

    def plus(self, w):
        v = self.v + w
        return Bounded(v, self.e + U * v.abs())

    def normed(self, kind, eps):
        v, e = self.v, self.e
        if kind is None:
            return self
        if kind == "layer":
            off = e.mean(-1, keepdim=True) + SUM * v.abs().mean(-1, keepdim=True) + 2 * U * v.mean(-1, keepdim=True).abs()
            v = v - v.mean(-1, keepdim=True)
            e = e + off + U * v.abs()
        power = (v * v).mean(-1, keepdim=True) + eps
        # of the factor: of the squares' sum (half of it), and what the values' errors make of the sum; a root, a quotient, a product, eps
        rel = SUM / 2 + 4 * U + ((v.abs() * e).mean(-1, keepdim=True) + (e * e).mean(-1, keepdim=True) / 2) / power
        r = power ** -0.5
        return Bounded(v * r, (e + v.abs() * rel) * r + U * (v * r).abs())


def gated_norm(x, f=None, post=None, post_gain=None, post_bias=None, post_eps=1e-5, gate=None, skip_scale=1.0, branch_scale=1.0, pre=None,
               pre_gain=None, pre_bias=None, pre_eps=1e-5, scale=None, shift=None, request=None):
    """(y, h) as Bounded; request [rows]: the row's vectors.  Scales and eps count as the fp32 numbers they become."""
    d = lambda t: None if t is None else t.double().cpu()
    f32 = lambda s: torch.tensor(float(s), dtype=torch.float32).double().item()
    at = lambda t: d(t) if request is None else d(t)[request]
    y = Bounded(d(x) * f32(skip_scale))
    y.e = U * y.v.abs()
    if f is not None:
        z = Bounded(d(f)).normed(post, f32(post_eps))
        if post_gain is not None:
            z = z.times(d(post_gain))
        if post_bias is not None:
            z = z.plus(d(post_bias))
        if gate is not None:
            z = z.times(at(gate))
        z = z.times(f32(branch_scale))
        v = z.v + y.v
        y = Bounded(v, z.e + y.e + U * v.abs())
    h = y.normed(pre, f32(pre_eps))
    if pre_gain is not None:
        h = h.times(d(pre_gain))
    if pre_bias is not None:
        h = h.plus(d(pre_bias))
    if scale is not None:
        h = h.times(1 + at(scale))
        h.e = h.e + U * h.v.abs()
    if shift is not None:
        h = h.plus(at(shift))
    return y, h


# ---- 8-bit floating point, from the definition
def f8_exponent(peak):
    """Smallest whole number of -100 .. 119 with peak <= 448 * 2^e (peak: 64 bits)."""
    e = torch.full_like(peak, -100.0)
    for k in range(-100, 119):
        e = torch.where(peak > 448.0 * 2.0 ** k, k + 1.0, e)
    return e


def f8_numbers():
    n = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8)]
    return torch.tensor(n[:-1], dtype=torch.float64)


def f8_round(v):
    """The nearest of the format's numbers, halves to the even one: of two neighbours in the list of all of them the one at an even place."""
    numbers = f8_numbers()
    a = v.abs().clamp(max=448.0)
    hi = torch.searchsorted(numbers, a.contiguous()).clamp(max=len(numbers) - 1)
    lo = (hi - 1).clamp(min=0)
    dl, dh = a - numbers[lo], numbers[hi] - a
    at = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return at, torch.where(v.signbit(), -numbers[at], numbers[at])


def f8_held(x):
    """x [rows, K] -> (bytes [rows, Kp], scale bytes [rows, Kp / 128], values held [rows, K]); NaN blocks hold NaN."""
    x = x.double().cpu()
    rows, K = x.shape
    Kp = -(-K // 128) * 128
    v = torch.zeros((rows, Kp), dtype=torch.float64)
    v[:, :K] = x
    v = v.view(rows, -1, 128)
    bad = ~torch.isfinite(v).all(-1, keepdim=True)
    v = torch.where(bad, torch.zeros_like(v), v)
    e = f8_exponent(v.abs().amax(-1, keepdim=True))
    e = torch.where(bad, torch.zeros_like(e), e)
    at, r = f8_round(v * 2.0 ** -e)
    code = at + torch.where(v.signbit(), 128, 0)
    code = torch.where(bad, torch.full_like(code, 127), code)
    held = torch.where(bad, torch.full_like(r, float("nan")), r * 2.0 ** e)
    return code.reshape(rows, Kp).to(torch.uint8), (e + 127).view(rows, -1).to(torch.uint8), held.reshape(rows, Kp)[:, :K].contiguous()


def linear_f8(x, w, b, res, dtype, device="cpu"):
    """(y, bound, size) of the layer: bound of every element's error, rounding included; size: magnitudes of the products, summed.
    bf16: of eight products of neighbouring K each loses less than 2^-13 of the largest, with numbers below the format's normal ones counting as the
    smallest of those.  Sums add (K / 16 + 32) times up to 2 U (the instruction cuts off) of the magnitudes summed."""
    hx, hw = f8_held(x)[2].to(device), f8_held(w.t().contiguous())[2].to(device)
    K = hx.shape[1]
    main, size = hx @ hw.t(), hx.abs() @ hw.abs().t()
    bound = (K / 16 + 32) * 2 * U * size
    if dtype == torch.bfloat16:
        def largest(h, src):
            scale = f8_held(src)[1].double().to(device) - 127
            low = (2.0 ** (scale - 6)).repeat_interleave(128, 1)
            v = torch.zeros((h.shape[0], low.shape[1]), dtype=torch.float64, device=device)
            v[:, :K] = h.abs()
            return torch.maximum(v, low).view(h.shape[0], -1, 8).amax(-1)
        bound = bound + 8 * 2.0 ** -13 * (largest(hx, x) @ largest(hw, w.t().contiguous()).t())
    want = main.clone()
    for t in (b, res):
        if t is not None:
            want = want + t.double().to(device)
            size = size + t.double().to(device).abs()
    bound = bound + 2 * U * size + HALF[dtype] * want.abs() + 1e-37
    return want, bound, size
