"""Plain 64-bit forms of the prompt-side operators (torch, CPU) and the error bounds their tests use.

u: half a step of fp32, H: half a step of the output type, both relative to the value.  Sums of n fp32 terms are counted with
2 n u (a matrix instruction may cut off instead of rounding)."""
import torch

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def steps(x):
    """(whole numbers, scale) of groups along the last axis: 127 x / amax to the nearest, halves to even."""
    x = x.double()
    amax = x.abs().amax(-1, keepdim=True)
    q = torch.where(amax > 0, torch.round(127 * x / torch.where(amax > 0, amax, torch.ones_like(amax))), torch.zeros_like(x))
    scale = amax / 127
    bad = ~torch.isfinite(amax)
    return torch.where(bad, torch.zeros_like(q), q), torch.where(bad, torch.full_like(scale, float("nan")), scale)


def held(x):
    q, s = steps(x)
    return q * s


def attention(q, k, v, scale, causal=True):
    """q [Lq, H, D], k, v [Lk, Hk, D] -> (out, |out| bound of the weights times |v|, largest sum of |q k| scale), 64 bits."""
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    (Lq, H, D), Lk, G = q.shape, k.shape[0], q.shape[1] // k.shape[1]
    out, bound, size = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((Lq, H, 1), dtype=torch.float64)
    for h in range(H):
        kh, vh = k[:, h // G], v[:, h // G]
        for i in range(Lq):
            n = max(0, min(Lk, i + Lk - Lq + 1)) if causal else Lk
            if n == 0:
                continue
            s = (kh[:n] @ q[i, h]) * scale
            p = torch.softmax(s, 0)
            out[i, h] = p @ vh[:n]
            bound[i, h] = p @ vh[:n].abs()
            size[i, h] = ((kh[:n].abs() @ q[i, h].abs()) * abs(scale)).max()
    return out, bound, size


def attention_tolerance(out, bound, size, dtype, D, Lk):
    """|error| of a row: scores off by (2 D + 4) u of their summed magnitudes (the 4: scale, its product, a key's scale, the
    subtraction of the reference) change a weight by the same share, twice (numerator and sum); exp2, the weights' sum and the output's:
    (2 Lk + 16) u; bf16 weights are rounded once; the result is rounded once."""
    share = 2 * (2 * D + 4) * U * size + (2 * 2 * Lk + 16) * U
    if dtype == torch.bfloat16:
        share = share + HALF[dtype]
    return share * bound + HALF[dtype] * out.abs() + 1e-30


def attention_by_heads(q, k, v, scale, causal=True):
    """`attention` a head at a time, on the tensors' device: for longer sequences."""
    q, k, v = q.double(), k.double(), v.double()
    (Lq, H, D), Lk, G = q.shape, k.shape[0], q.shape[1] // k.shape[1]
    out, bound, size = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((Lq, H, 1), dtype=torch.float64, device=q.device)
    seen = torch.ones((Lq, Lk), dtype=torch.bool, device=q.device)
    if causal:
        seen = seen.tril(Lk - Lq)
    some = seen.any(1, keepdim=True)
    for h in range(H):
        kh, vh = k[:, h // G].contiguous(), v[:, h // G].contiguous()
        s = (q[:, h].contiguous() @ kh.t().contiguous()) * scale
        p = torch.softmax(s.masked_fill(~seen, float("-inf")), 1)
        p = torch.where(some, p, torch.zeros_like(p))
        out[:, h], bound[:, h] = p @ vh, p @ vh.abs()
        size[:, h] = ((q[:, h].abs().contiguous() @ kh.abs().t().contiguous()) * abs(scale)).masked_fill(~seen, 0.0).amax(1, keepdim=True)
    return out, bound, size
