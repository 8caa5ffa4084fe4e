"""64-bit form of the prompt attention for scores that are not finite, and error bounds that know how a path rounds its weights.

u: half a step of fp32, H: half a step of the output's type, both relative to the value."""
import torch

from prompt_oracle import HALF, U

ONE_PIECE, TWO_PIECES = 2.0 ** -8, 2.0 ** -16       # what a weight loses as one bf16 number, as two that add up to it


def attention(q, k, v, scale, causal=True):
    """q [Lq, H, D], k, v [Lk, Hk, D], the queries at the end of the keys, in 64 bits on the tensors' device.  A score of +infinity or
    NaN makes its row NaN, one of -infinity weighs nothing, a row without another score is 0.  -> out, the weights times |v|, the
    norm of the weighted values taken one by one, the largest sum of |q k| |scale| among the finite keys."""
    q, k, v = q.double(), k.double(), v.double()
    (Lq, H, D), Lk, G = q.shape, k.shape[0], q.shape[1] // k.shape[1]
    out, bound, spread = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    size = torch.zeros((Lq, H, 1), dtype=torch.float64, device=q.device)
    seen = torch.ones((Lq, Lk), dtype=torch.bool, device=q.device)
    if causal:
        seen = seen.tril(Lk - Lq)
    low = torch.full((), float("-inf"), dtype=torch.float64, device=q.device)
    if Lk == 0:
        return out, bound, spread, size
    for h in range(H):
        kh, vh, qh = k[:, h // G].contiguous(), v[:, h // G].contiguous(), q[:, h].contiguous()
        s = torch.where(seen, (qh @ kh.t().contiguous()) * scale, low)
        bad = (s.isnan() | (s == float("inf"))).any(1, keepdim=True)
        top = s.amax(1, keepdim=True)
        w = torch.where(s == low, torch.zeros_like(s), torch.exp(s - torch.where(top == low, torch.zeros_like(top), top)))
        total = w.sum(1, keepdim=True)
        p = torch.where(total == 0, torch.zeros_like(w), w / total)
        p = torch.where(bad, torch.full_like(p, float("nan")), p)
        out[:, h], bound[:, h], spread[:, h] = p @ vh, p @ vh.abs(), ((p * p) @ (vh * vh)).sqrt()
        finite = torch.where(kh.isfinite(), kh, torch.zeros_like(kh))
        size[:, h] = ((qh.abs() @ finite.abs().t().contiguous()) * abs(scale)).masked_fill(~seen, 0.0).amax(1, keepdim=True)
    return out, bound, spread, size


def tolerance(out, bound, size, dtype, D, Lk, piece, scales=0):
    """|error| of an element: scores off by (2 D + 4) u of their summed magnitudes (the 4: scale, its product, a key's scale, the
    subtraction of the reference) change a weight by the same share, twice (numerator and sum); exp2, the weights' sum and the
    output's: (4 Lk + 16) u; bf16: a weight loses `piece` of itself on its way to the matrix cores; `scales` u for what a value's scale adds;
    the result is rounded once."""
    share = 2 * (2 * D + 4) * U * size + (4 * Lk + 16 + scales) * U + (piece if dtype == torch.bfloat16 else 0.0)
    return share * bound + HALF[dtype] * out.abs() + 1e-30


def norm_bound(out, bound, spread, size, dtype, D, Lk, piece):
    """Norm of the error of all elements, with the roundings of the keys' weights and of the sums' steps taken as independent (they
    are thousands): what a weight loses adds up as the norm of the weighted values, the steps of a sum as the root of their number, both
    within a factor of 1.7 (sqrt(3): half a step against its root mean square) and more of what is expected.  The result's own rounding counts in full."""
    weights = 2 * (2 * D + 4) * U * size.max() + (piece if dtype == torch.bfloat16 else 0.0) + 16 * U
    return HALF[dtype] * out.norm() + weights * spread.norm() + 4 * (Lk ** 0.5) * U * bound.norm()
