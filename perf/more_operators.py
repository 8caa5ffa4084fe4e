"""Performance cases of the layer-side operators: rotary positions with several axes, norms before and after a sub-layer with its
gate and residual scale, and linear layers in 8-bit floating point with a scale for each block of 128.

What a transformer layer over image, video and text tokens needs around its attention: the sub-layer's input is normalised and
modulated (and rounded to 8 bits for the product behind it), queries and keys are turned by their positions, and the sub-layer's
output comes back through a norm, a gate and the residual.

  op        "rotary"  pserve_rotary: queries and keys turned by positions on up to three axes
            "norm"    pserve_gated_norm: what ends one sub-layer and begins the next, in one pass
            "linear"  pserve_linear_f8: rows rounded to 8 bits in blocks of 128, products, bias, residual
            "feed"    pserve_gated_norm into 8-bit rows, pserve_linear_f8 on them
  dtype     "bf16" or "f32"
  tokens, heads, kv_heads, dim, pairs     rotary: head layout, pairs of values on each axis ("t,h,w")
  layout    "half" (pair i: values i and i + P of a head, P pairs) or "next" (2 i and 2 i + 1)
  shared    one ladder of frequencies over all pairs, or one for each axis
  grid      "HxW" of the frames the tokens fill one after another; "" for single tokens far behind
  rows, C, requests, post, pre, mod       norm: kinds "rms", "layer" or "" behind and in front of a sub-layer, per-request vectors
  rows, K, N, res                         a linear layer

Where `own` is false `run` computes the operators in elementary torch operations in 32 bits (angles in 64); where it is true it
calls the framework.
"""
import math

import torch

own = False


# ------------------------------------------------------------------------------------------------ the cases
def _rotary(name, tokens, heads, kv_heads, dim, pairs, layout="half", shared=False, grid="", dtype="bf16"):
    return _named(name, dict(op="rotary", dtype=dtype, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, pairs=pairs, layout=layout,
                             shared=shared, grid=grid))


def _norm(name, rows, C, requests, post, pre, mod, dtype="bf16"):
    return _named(name, dict(op="norm", dtype=dtype, rows=rows, C=C, requests=requests, post=post, pre=pre, mod=mod))


def _linear(name, rows, K, N, res=False, dtype="bf16"):
    return _named(name, dict(op="linear", dtype=dtype, rows=rows, K=K, N=N, res=res))


def _feed(name, rows, C, N, requests, post, pre, mod):
    return _named(name, dict(op="feed", dtype="bf16", rows=rows, C=C, N=N, requests=requests, post=post, pre=pre, mod=mod))


def _named(name, case):
    return dict(case, name=name) if name else case


def listed():
    return [
        # one decoding step of 48 sequences far behind their prompts, grouped heads: all of it latency
        _rotary("rotary_step_48", 48, 32, 8, 128, "16,24,24", shared=True),
        # the tokens of a batch of the joint model, queries and keys inside one q/k/v matrix, neighbouring values paired
        _rotary("rotary_joint_12544", 12544, 24, 24, 64, "8,12,12", layout="next", grid="64x64"),
        # the skewed batch's 131,072 tokens at 640 channels
        _rotary("rotary_image_131k", 131072, 10, 10, 64, "8,12,12", grid="256x256"),
        # 32-bit inference over frames of odd size, a head width that is no power of two and not turned to its end
        _rotary("rotary_f32_partial", 5005, 12, 4, 80, "8,12,12", grid="35x13", dtype="f32"),
        # a decoding step of 32 sequences, between two sub-layers
        _norm("norm_step_32", 32, 4096, 1, "rms", "rms", False),
        # the joint model's tokens, gate behind one sub-layer, scale and shift in front of the next
        _norm("norm_joint_12544", 12544, 1536, 22, "rms", "layer", True),
        # 32-bit inference, a width that no tile divides
        _norm("norm_f32_odd", 1694, 1000, 7, "layer", "rms", True, dtype="f32"),
        # a linear layer of a decoding step: twelve rows, all of it reading weights
        _linear("linear_f8_step_12", 12, 4096, 4096),
        # a layer over 22 prompts in 32 bits, widths that no tile divides, with its residual
        _linear("linear_f8_f32_odd", 1694, 1000, 2500, res=True, dtype="f32"),
        # the largest layer of the joint model, with its residual
        _linear("linear_f8_12544", 12544, 1536, 6144, res=True),
        # one sub-layer's end, the next one's norm in 8 bits, its q/k/v layer
        _feed("feed_12544", 12544, 1536, 4608, 22, "rms", "layer", True),
        # the same for a short batch
        _feed("feed_333", 333, 640, 1920, 5, "", "layer", True),
    ]


def draw(rng):
    def some(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def width(lo, hi):
        x = some(lo, hi)
        return max(64, x // 64 * 64) if rng.random() < 0.7 else x

    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    size = 2 if dtype == "bf16" else 4
    op = rng.choice(["rotary", "rotary", "rotary", "norm", "norm", "norm", "linear", "linear", "feed"])
    if op == "rotary":
        kv_heads = rng.choice([1, 2, 4, 8, 8, 12])
        heads = kv_heads * rng.choice([1, 1, 2, 3, 4])
        dim = rng.choice([64, 64, 128, 128, 128, 32, 80, 96])
        t = rng.choice([dim // 8, dim // 8, dim // 16])
        h = rng.choice([dim // 8, 3 * dim // 16])
        w = min(dim // 2 - t - h, h)
        step = rng.random() < 0.35
        most = int(131072 * 20 * 64 * 2 / (size * dim * (heads + kv_heads)))
        tokens = some(1, 128) if step else some(65, min(200000, most))
        grid = "" if step else "%dx%d" % (some(4, 256), some(4, 256))
        return _rotary("", tokens, heads, kv_heads, dim, "%d,%d,%d" % (t, h, w), rng.choice(["half", "next"]), rng.random() < 0.5, grid, dtype)
    post, pre = rng.choice([("rms", "rms"), ("rms", "layer"), ("layer", "rms"), ("", "layer"), ("rms", "")])
    mod = rng.random() < 0.7
    if op == "norm":
        C = width(64, 8192)
        rows = some(1, max(1, min(65536, 12544 * 1536 * 2 // (C * size))))
        return _norm("", rows, C, rng.choice([1, 3, 22, 100]) if mod else 1, post, pre, mod, dtype)
    if op == "feed":
        C, N = width(64, 4096), width(64, 6144)
        rows = some(1, max(1, min(16384, int(8.8e10 / C / N))))
        return _feed("", rows, C, N, rng.choice([1, 3, 22]) if mod else 1, post, pre or "rms", mod)
    K, N = width(64, 8192), width(64, 8192)
    rows = some(1, max(1, min(16384, int(1.1e11 / K / N / (1 if dtype == "bf16" else 4)))))
    return _linear("", rows, K, N, rng.random() < 0.5, dtype)


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _ladders(case):
    """(axis, frequency) of every pair: steps from 1 down towards 1 / 10000 over all pairs, or over each axis' own."""
    pairs = [int(p) for p in case["pairs"].split(",")]
    axis = [a for a, n in enumerate(pairs) for _ in range(n)]
    if case["shared"]:
        return axis, [10000.0 ** (-i / len(axis)) for i in range(len(axis))]
    return axis, [10000.0 ** (-i / n) for n in pairs for i in range(n)]


class _Inputs:
    """Everything random of a case, drawn from the seed on the GPU: queries and keys as projections of normalised activations are
    (normal), keys with a few channels that stand out; token rows whose sizes differ, a few channels that stand out; gains
    around 1, gates and modulations as a conditioning vector gives them; weights of variance 1 / fan-in."""

    def __init__(self, case, seed):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        dt = _dtype(case)

        def normal(*shape):
            return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

        op = case["op"]
        if op == "rotary":
            T, H, Hk, D = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
            if H == Hk:                                     # queries, keys and values of one projection
                qkv = normal(T, 3 * H, D).to(dt)
                self.q, self.k = qkv[:, :H], qkv[:, H:2 * H]
            else:
                self.q = normal(T, H, D).to(dt)
                self.k = (normal(T, Hk, D) * torch.exp(0.4 * normal(Hk, D))).to(dt)
            if case["grid"]:
                h, w = (int(x) for x in case["grid"].split("x"))
                i = torch.arange(T, device="cuda")
                first = torch.randint(0, 64, (3,), generator=gen, device="cuda")
                at = torch.stack([i // (h * w), i // w % h, i % w], 1) + first
            else:
                at = torch.randint(0, 1 << 17, (T, 1), generator=gen, device="cuda").expand(T, 3)
            self.pos = at.float().contiguous()
            return
        if op == "linear":
            rows, K, N = case["rows"], case["K"], case["N"]
            self.x = (normal(rows, K) * torch.exp(0.5 * normal(rows, 1))).to(dt)
            self.res = normal(rows, N).to(dt) if case["res"] else None
        else:
            rows, K, n = case["rows"], case["C"], case["requests"]
            N = case.get("N", 0)
            channel = torch.exp(0.4 * normal(K))
            self.x = (normal(rows, K) * torch.exp(0.3 * normal(rows, 1)) * channel).to(dt)
            self.f = (2 * normal(rows, K) * torch.exp(0.5 * normal(rows, 1))).to(dt)
            self.post_gain = (1 + 0.2 * normal(K)).to(dt) if case["post"] else None
            self.pre_gain = (1 + 0.2 * normal(K)).to(dt) if case["pre"] == "rms" or not case["mod"] and case["pre"] else None
            self.pre_bias = (0.1 * normal(K)).to(dt) if self.pre_gain is not None and case["pre"] == "layer" else None
            self.mod = (0.3 * normal(n, 3 * K)).to(dt) if case["mod"] else None     # gate, scale, shift of every request
            cut = torch.randint(0, rows + 1, (n - 1,), generator=gen, device="cuda").sort().values
            ends = torch.tensor([0, rows], device="cuda")
            self.cu = torch.cat([ends[:1], cut, ends[1:]]).int()
        if N:
            self.w = (normal(K, N) / math.sqrt(K)).to(dt)
            self.b = (0.1 * normal(N)).to(dt)


_BRANCH = 0.7


class _State:
    pass


def prepare(case, seed):
    i = _Inputs(case, seed)
    s = _State()
    s.case, s.own = case, own
    op = case["op"]
    code = None
    if own:
        import paper_2501_09253_amd as ps
        code = ps.BF16 if case["dtype"] == "bf16" else ps.F32
    if op == "rotary":
        s.q, s.k, s.pos = i.q, i.k, i.pos
        axis, freq = _ladders(case)
        if own:
            s.rotary = ps.Rotary(axis, freq, layout=case["layout"])
        else:
            s.axis = torch.tensor(axis, device="cuda")
            s.freq = torch.tensor(freq, dtype=torch.float64, device="cuda")
        return s
    if op == "linear":
        s.x, s.res = i.x, i.res
    else:
        s.x, s.f, s.cu = i.x, i.f, i.cu
        s.post_gain, s.pre_gain, s.pre_bias = i.post_gain, i.pre_gain, i.pre_bias
        s.gate = s.scale = s.shift = None
        if i.mod is not None:
            s.gate, s.scale, s.shift = i.mod.chunk(3, dim=1)
    if op != "norm":
        if own:
            s.layer = ps.LinearF8(i.w, i.b, code)
            if op == "feed":
                s.rows8 = ps.RowsF8(case["rows"], case["C"])
        else:
            s.w, s.b = _blocks(i.w.t().float()), i.b.float()
    return s


# ------------------------------------------------------------------------------------------------ the plain forms
def _blocks(x):
    """The values that x [rows, K] stands for in 8 bits: blocks of 128 along K share a power of two, the smallest with which no
    value of the block passes 448 (2^-100 .. 2^119); each value is the nearest number of three fraction bits and exponents from -6."""
    rows, K = x.shape
    pad = torch.zeros((rows, -K % 128), dtype=torch.float32, device=x.device)
    v = torch.cat([x, pad], 1).view(rows, -1, 128)
    fraction, exponent = torch.frexp(v.abs().amax(-1, keepdim=True))
    shift = (exponent - 9 + (fraction > 0.875).int()).clamp(-100, 119)      # 448 = 0.875 * 2^9
    v = torch.ldexp(v, -shift)
    step = torch.ldexp(torch.ones_like(v), torch.frexp(v).exponent.clamp(min=-5) - 4)
    return torch.ldexp(torch.round(v / step) * step, shift).view(rows, -1)[:, :K].contiguous()


def _normed(x, kind, eps=1e-5):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    if kind:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
    return x


def _join(s):
    """(end of one sub-layer, beginning of the next) in 32 bits."""
    request = torch.searchsorted(s.cu, torch.arange(s.x.shape[0], dtype=torch.int32, device="cuda"), right=True) - 1
    z = _normed(s.f.float(), s.case["post"])
    if s.post_gain is not None:
        z = z * s.post_gain.float()
    if s.gate is not None:
        z = z * s.gate.float()[request]
    y = s.x.float() + _BRANCH * z
    if not s.case["pre"]:
        return y, None
    h = _normed(y, s.case["pre"])
    if s.pre_gain is not None:
        h = h * s.pre_gain.float()
    if s.pre_bias is not None:
        h = h + s.pre_bias.float()
    if s.scale is not None:
        h = h * (1 + s.scale.float()[request]) + s.shift.float()[request]
    return y, h


def _turn(s, x, cos, sin):
    P, D = cos.shape[1], x.shape[2]
    x = x.float()
    even, odd = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if s.case["layout"] == "next" else (slice(0, P), slice(P, 2 * P))
    out = torch.empty(x.shape, dtype=torch.float32, device=x.device)
    a, b = x[..., even], x[..., odd]
    out[..., even] = a * cos[:, None] - b * sin[:, None]
    out[..., odd] = a * sin[:, None] + b * cos[:, None]
    if 2 * P < D:
        out[..., 2 * P:] = x[..., 2 * P:]
    return out


def _plain(s):
    op, dt = s.case["op"], _dtype(s.case)
    if op == "rotary":
        angle = s.pos.double()[:, s.axis] * s.freq
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
        return [_turn(s, s.q, cos, sin).to(dt), _turn(s, s.k, cos, sin).to(dt)]
    if op == "norm":
        return [t.to(dt) for t in _join(s) if t is not None]
    if op == "feed":
        y, h = _join(s)
        return [y.to(dt), (torch.matmul(_blocks(h), s.w.t()) + s.b).to(dt)]
    y = torch.matmul(_blocks(s.x.float()), s.w.t()) + s.b
    return (y if s.res is None else y + s.res.float()).to(dt)


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    if not s.own:
        return _plain(s)
    import paper_2501_09253_amd as ps
    op = s.case["op"]
    if op == "rotary":
        return list(s.rotary.forward(s.q, s.k, s.pos))
    if op == "linear":
        return s.layer.forward(s.x, res=s.res)
    kinds = dict(post=s.case["post"] or None, post_gain=s.post_gain, gate=s.gate, branch_scale=_BRANCH, pre=s.case["pre"] or None,
                 pre_gain=s.pre_gain, pre_bias=s.pre_bias, scale=s.scale, shift=s.shift, cu_rows=s.cu)
    if op == "norm":
        if not s.case["pre"]:                               # the end of a last sub-layer: nothing behind it
            kinds.update(scale=None, shift=None)
        return [t for t in ps.gated_norm(s.x, s.f, **kinds) if t is not None]
    y, _ = ps.gated_norm(s.x, s.f, rows8=s.rows8, **kinds)
    return [y, s.layer.forward(s.rows8)]


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    op = case["op"]
    if op == "rotary":
        values = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["dim"]
        return {"bytes": 2 * values * size + 12 * case["tokens"], "flops": 3 * values}
    if op == "linear":
        rows, K, N = case["rows"], case["K"], case["N"]
        return {"bytes": rows * K * size + K * N + K * N // 128 + rows * N * size * (2 if case["res"] else 1) + N * size,
                "flops": 2 * rows * K * N}
    rows, C = case["rows"], case["C"]
    vectors = (3 * case["requests"] * C if case["mod"] else 0) + 2 * C
    if op == "norm":
        behind = bool(case["pre"])
        return {"bytes": rows * C * size * (4 if behind else 3) + vectors * size, "flops": rows * C * (6 + (6 if behind else 0))}
    N = case["N"]
    return {"bytes": 3 * rows * C * size + vectors * size + C * N + C * N // 128 + rows * N * size, "flops": 2 * rows * C * N + 12 * rows * C}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _e4m3_64():
    """All numbers of the 8-bit format that are not negative, ascending."""
    small = [m * 2.0 ** -9 for m in range(8)]
    return torch.tensor(small + [(8 + m) * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8)][:-1], dtype=torch.float64, device="cuda")


def _held64(x):
    """The values that rows of x (64 bits) stand for in 8 bits, by a search among the format's numbers."""
    numbers = _e4m3_64()
    border = (numbers[1:] + numbers[:-1]) / 2
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], 128):
        part = x[:, c:c + 128]
        peak = part.abs().max(1, keepdim=True).values
        e = torch.ceil(torch.log2(peak / 448)).clamp(-100, 119)
        e = torch.where(peak > 448 * torch.exp2(e), e + 1, e)               # (the logarithm's rounding)
        e = torch.where((peak <= 448 * torch.exp2(e - 1)) & (e > -100), e - 1, e)
        v = part / torch.exp2(e)
        at = torch.searchsorted(border, v.abs().contiguous())               # a value on a border: the number below it
        up = (at < border.numel()) & (v.abs() == border[at.clamp(max=border.numel() - 1)]) & (at % 2 == 1)
        out[:, c:c + 128] = torch.sign(v) * numbers[at + up.long()] * torch.exp2(e)
    return out


def exact(case, seed):
    i = _Inputs(case, seed)
    op, d = case["op"], torch.float64
    if op == "rotary":
        axis, freq = _ladders(case)
        turn = torch.stack([i.pos[:, a].to(d) * f for a, f in zip(axis, freq)], 1)
        turn = torch.polar(torch.ones_like(turn), turn)[:, None]            # e^(i theta)
        P, outs = len(axis), []
        for x in (i.q, i.k):
            x = x.to(d)
            if case["layout"] == "next":
                z = torch.view_as_complex(x[..., :2 * P].reshape(*x.shape[:2], P, 2).contiguous()) * turn
                head = torch.view_as_real(z).reshape(*x.shape[:2], 2 * P)
            else:
                z = torch.complex(x[..., :P].contiguous(), x[..., P:2 * P].contiguous()) * turn
                head = torch.cat([z.real, z.imag], -1)
            outs.append(torch.cat([head, x[..., 2 * P:]], -1))
        return outs
    if op != "linear":
        def norm(v, kind):
            if kind == "layer":
                return (v - v.mean(1, keepdim=True)) / torch.sqrt(v.var(1, correction=0, keepdim=True) + 1e-5)
            return v / torch.sqrt(v.square().sum(1, keepdim=True) / v.shape[1] + 1e-5) if kind == "rms" else v

        y = torch.empty(i.x.shape, dtype=d, device="cuda")
        h = torch.empty_like(y)
        cu = i.cu.tolist()
        for r in range(len(cu) - 1):
            a, b = cu[r], cu[r + 1]
            if a == b:
                continue
            gate, scale, shift = (0, 0, 0) if i.mod is None else i.mod[r].to(d).chunk(3)
            branch = norm(i.f[a:b].to(d), case["post"])
            branch = branch * (1 if i.post_gain is None else i.post_gain.to(d)) * (1 if i.mod is None else gate)
            y[a:b] = i.x[a:b].to(d) + _BRANCH * branch
            g = norm(y[a:b], case["pre"]) * (1 if i.pre_gain is None else i.pre_gain.to(d)) + (0 if i.pre_bias is None else i.pre_bias.to(d))
            h[a:b] = g * (1 + scale) + shift
        if op == "norm":
            return [y, h] if case["pre"] else [y]
        return [y, torch.mm(_held64(h), _held64(i.w.to(d).t().contiguous()).t().contiguous()) + i.b.to(d)]
    out = torch.mm(_held64(i.x.to(d)), _held64(i.w.to(d).t().contiguous()).t().contiguous()) + i.b.to(d)
    return out if i.res is None else out + i.res.to(d)
