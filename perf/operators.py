"""Performance cases of the prompt-side operators: causal attention over packed prompts, the 8-bit key/value store with the
attention that reads it, and linear layers in 8-bit integers.

What stands beside the denoising block on a server's GPU: the causal text transformer that turns the prompts of a batch into the
text rows of the block, and the one that extends short prompts token by token.

  op        "attn"    pserve_prompt_attention: keys and values as packed tensors
            "store"   the 8-bit store: write the keys and values of new tokens, read them back
            "cached"  pserve_kv8_attention: keys and values in pages of the 8-bit store
            "linear"  pserve_linear8: tokens quantised row by row, 8-bit products, bias, residual
  dtype     "bf16" or "f32"
  lens      tokens of each sequence ("new+old" in "cached": new queries behind old keys), "a,b*count,..."
  heads, kv_heads, dim      head layout
  page      tokens of a page ("cached", "store")
  rows, K, N, res           a linear layer

Where `own` is false `run` computes the operators in elementary torch operations in 32 bits (the 8-bit rounding in 64, where a
quotient can lie at the border of two steps); where it is true it calls the framework.
"""
import math

import torch

own = False


# ------------------------------------------------------------------------------------------------ the cases
def _attn(name, lens, heads, kv_heads, dim, dtype="bf16"):
    return _named(name, dict(op="attn", dtype=dtype, lens=lens, heads=heads, kv_heads=kv_heads, dim=dim))


def _store(name, tokens, kv_heads, dim, page=64, dtype="bf16"):
    return _named(name, dict(op="store", dtype=dtype, tokens=tokens, kv_heads=kv_heads, dim=dim, page=page))


def _cached(name, lens, heads, kv_heads, dim, page=64, dtype="bf16"):
    return _named(name, dict(op="cached", dtype=dtype, lens=lens, heads=heads, kv_heads=kv_heads, dim=dim, page=page))


def _linear(name, rows, K, N, res=False, dtype="bf16"):
    return _named(name, dict(op="linear", dtype=dtype, rows=rows, K=K, N=N, res=res))


def _named(name, case):
    return dict(case, name=name) if name else case


def listed():
    return [
        # the text encoder over the prompts of 22 requests, 77 tokens each: a short call, all of it latency
        _attn("attn_text_22x77", "77*22", 12, 12, 64),
        # prompts of a mixed batch as they came, templates and long descriptions, grouped heads
        _attn("attn_ragged_gqa", "31,2211,77*6,640,1024,1535,154*4,333,4096,18,905,1,2700", 32, 8, 128),
        # one long document as a prompt
        _attn("attn_long_16k", "16384", 32, 8, 128),
        # 32-bit inference, a head width that is no power of two, odd lengths
        _attn("attn_f32_odd", "1,77,300,511,1000,77", 8, 2, 80, dtype="f32"),
        # one decoding step of 48 sequences: their new keys and values into the store (and back)
        _store("store_step_48", 48, 8, 128),
        # a prompt batch's keys and values into the store and back
        _store("store_prompts_20k", 20011, 8, 128),
        # one decoding step: 32 sequences of very different length, a query token each
        _cached("decode_32", "1+500*8,1+1023*6,1+77*6,1+2048*4,1+3500*4,1+7999*3,1+12", 32, 8, 128),
        # one decoding step of a single very long sequence in small pages
        _cached("decode_1x131k", "1+131071", 32, 8, 128, page=16),
        # four prompts extended by some hundred tokens behind what the store already holds
        _cached("extend_4", "512+3583,300+1200,640+2048,77+640", 16, 4, 64),
        # a linear layer of a decoding step: twelve rows, all of it reading weights
        _linear("linear_step_12", 12, 4096, 4096),
        # a layer over the 22 prompts in 32 bits, widths that no tile divides
        _linear("linear_f32_odd", 1694, 1000, 2500, res=True, dtype="f32"),
        # the largest layer of the transformer model's level, with its residual
        _linear("linear_12544", 12544, 1536, 6144, res=True),
    ]


def draw(rng):
    def log_uniform(lo, hi):
        return math.exp(rng.uniform(math.log(lo), math.log(hi)))

    def some(lo, hi):
        return max(lo, min(hi, int(round(log_uniform(lo, hi)))))

    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 12])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 8])
    dim = rng.choice([64, 64, 128, 128, 128, 32, 80, 96])
    op = rng.choice(["attn", "attn", "store", "cached", "cached", "linear", "linear"])
    if op == "attn":
        # pairs of queries and keys are held below those of the largest listed case
        n = some(1, 32)
        top = 12000 if dtype == "bf16" else 3000
        lens, left = [], 1.2e8 * 32 * 128 / (heads * dim) / (1 if dtype == "bf16" else 16)
        for _ in range(n):
            x = some(1, top)
            x = max(1, min(x, int(math.sqrt(2 * left / n))))
            lens.append(x)
        return _attn("", ",".join(map(str, lens)), heads, kv_heads, dim, dtype)
    if op == "store":
        most = 20000 * 8 * 128 // (kv_heads * dim) // (1 if dtype == "bf16" else 2)
        return _store("", some(1, most), kv_heads, dim, rng.choice([16, 64, 256]), dtype)
    if op == "cached":
        n = some(1, 48)
        step = rng.random() < 0.6
        most = 131072 * 8 * 128 // (kv_heads * dim) // n // (1 if dtype == "bf16" else 4)
        most = max(1, min(131072, most))
        parts = []
        for _ in range(n):
            old = some(1, most)
            new = rng.choice([1, 1, 1, 2, 4]) if step else some(1, 512 if n <= 8 else 64)
            parts.append("%d+%d" % (new, old))
        return _cached("", ",".join(parts), heads, kv_heads, dim, rng.choice([16, 32, 64, 128]), dtype)
    K, N = some(64, 8192), some(64, 8192)
    if rng.random() < 0.7:
        K, N = max(64, K // 64 * 64), max(64, N // 64 * 64)
    most = max(1, min(16384, int(1.1e11 / K / N / (1 if dtype == "bf16" else 4))))
    return _linear("", some(1, most), K, N, rng.random() < 0.5, dtype)


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lens(case):
    """(new, old) tokens of every sequence."""
    out = []
    for part in case["lens"].split(","):
        one, _, count = part.partition("*")
        new, _, old = one.partition("+")
        out += [(int(new), int(old or 0))] * int(count or 1)
    return out


def _starts(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class _Inputs:
    """Everything random of a case, drawn from the seed on the GPU: queries, keys and values as projections of normalised
    activations are (normal), keys with a few channels that stand out; rows of a layer with token sizes that differ; weights of
    variance 1 / fan-in."""

    def __init__(self, case, seed):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        dt = _dtype(case)

        def normal(shape):
            return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

        op = case["op"]
        if op == "linear":
            rows, K, N = case["rows"], case["K"], case["N"]
            self.x = (normal((rows, K)) * torch.exp(0.5 * normal((rows, 1)))).to(dt)
            self.w = (normal((K, N)) / math.sqrt(K)).to(dt)
            self.b = (0.1 * normal((N,))).to(dt)
            self.res = normal((rows, N)).to(dt) if case["res"] else None
            return
        Hk, D = case["kv_heads"], case["dim"]

        def keys(tokens):
            return (normal((tokens, Hk, D)) * torch.exp(0.4 * normal((Hk, D)))).to(dt)

        if op == "store":
            t, page = case["tokens"], case["page"]
            self.k, self.v = keys(t), normal((t, Hk, D)).to(dt)
            self.pages = -(-t // page) + 8
            order = torch.randperm(self.pages, generator=gen, device="cuda")
            place = torch.arange(t, device="cuda")
            self.places = order[place // page] * page + place % page
            return
        self.lens = _lens(case)
        self.cu_q = _starts([new for new, _ in self.lens])
        self.cu_k = _starts([new + old for new, old in self.lens])
        self.q = normal((self.cu_q[-1], case["heads"], D)).to(dt)
        self.k = keys(self.cu_k[-1])
        self.v = normal((self.cu_k[-1], Hk, D)).to(dt)
        if op == "cached":
            page = case["page"]
            used = [-(-(new + old) // page) for new, old in self.lens]
            self.pages = sum(used) + 4
            order = torch.randperm(self.pages, generator=gen, device="cuda")
            self.table = torch.zeros((len(used), max(used)), dtype=torch.int32, device="cuda")
            self.places = torch.empty(self.cu_k[-1], dtype=torch.int64, device="cuda")
            for s, (u, at) in enumerate(zip(used, _starts(used))):
                self.table[s, :u] = order[at:at + u].int()
                j = torch.arange(self.cu_k[s + 1] - self.cu_k[s], device="cuda")
                self.places[self.cu_k[s]:self.cu_k[s + 1]] = self.table[s].long()[j // page] * page + j % page


class _State:
    pass


def prepare(case, seed):
    i = _Inputs(case, seed)
    s = _State()
    s.case, s.own = case, own
    op = case["op"]
    if op == "linear":
        s.x, s.b, s.res = i.x, i.b, i.res
        if own:
            import paper_2501_09253_amd as ps
            s.layer = ps.Linear8(i.w, i.b, ps.BF16 if case["dtype"] == "bf16" else ps.F32)
            s.y = torch.empty((case["rows"], case["N"]), dtype=i.x.dtype, device="cuda")
        else:
            s.w8, s.w_scale = _to_8bit(i.w.t().contiguous())
        return s
    Hk, D = case["kv_heads"], case["dim"]
    if op == "store":
        s.k, s.v, s.places = i.k, i.v, i.places
        if own:
            import paper_2501_09253_amd as ps
            s.store = ps.KV8(i.pages * case["page"], Hk, D)
        else:
            s.held = _empty_store(i.pages * case["page"], Hk, D)
        return s
    s.q, s.lens = i.q, i.lens
    s.cu_q, s.cu_k = _int32(i.cu_q), _int32(i.cu_k)
    s.max_q, s.max_k = max(new for new, _ in i.lens), max(new + old for new, old in i.lens)
    if op == "attn":
        s.k, s.v = i.k, i.v
        return s
    s.table, s.page = i.table, case["page"]
    s.key_len = s.cu_k[1:] - s.cu_k[:-1]
    if own:
        import paper_2501_09253_amd as ps
        s.store = ps.KV8(i.pages * s.page, Hk, D)
        s.store.write(i.k, i.v, i.places)
    else:
        s.held = _empty_store(i.pages * s.page, Hk, D)
        _write(s.held, i.k, i.v, i.places)
    return s


# ------------------------------------------------------------------------------------------------ the plain forms
def _to_8bit(x):
    """Whole numbers of -127 .. 127 and the scale of every row (the last axis)."""
    x64 = x.double()
    most = x64.abs().amax(-1, keepdim=True)
    q = torch.where(most > 0, torch.round(x64 * 127 / torch.where(most > 0, most, 1.0)), 0.0)
    return q.to(torch.int8), (most / 127).float()


def _empty_store(places, heads, dim):
    held = {}
    for name in ("k", "v"):
        held[name] = torch.zeros((places, heads, dim), dtype=torch.int8, device="cuda")
        held[name + "_scale"] = torch.zeros((places, heads, 1), dtype=torch.float32, device="cuda")
    return held


def _write(held, k, v, places):
    for name, x in (("k", k), ("v", v)):
        q, scale = _to_8bit(x)
        held[name][places] = q
        held[name + "_scale"][places] = scale


def _read(held, places):
    return [held[name][places].float() * held[name + "_scale"][places] for name in ("k", "v")]


def _attention(q, k, v, scale):
    """Queries [Lq, H, D] at the end of the keys [Lk, Hk, D], in 32 bits; some of the queries at a time."""
    Lq, H, D = q.shape
    Lk, Hk, _ = k.shape
    kt = k.float().permute(1, 2, 0).contiguous().unsqueeze(1)            # [Hk, 1, D, Lk]
    vt = v.float().permute(1, 0, 2).contiguous().unsqueeze(1)            # [Hk, 1, Lk, D]
    out = torch.empty((Lq, H, D), dtype=torch.float32, device=q.device)
    step = max(1, min(Lq, (1 << 28) // max(1, H * Lk)))
    column = torch.arange(Lk, device=q.device)
    for a in range(0, Lq, step):
        b = min(Lq, a + step)
        rows = q[a:b].float().reshape(b - a, Hk, H // Hk, D).permute(1, 2, 0, 3).contiguous()
        score = torch.matmul(rows, kt) * scale
        ahead = column[None, :] > torch.arange(a, b, device=q.device)[:, None] + (Lk - Lq)
        score.masked_fill_(ahead, float("-inf"))
        score -= score.amax(-1, keepdim=True)
        score.exp_()
        total = score.sum(-1, keepdim=True)
        o = torch.matmul(score, vt) / total
        out[a:b] = o.permute(2, 0, 1, 3).reshape(b - a, H, D)
    return out


def _plain(s):
    case = s.case
    op = case["op"]
    if op == "linear":
        x8, x_scale = _to_8bit(s.x)
        y = torch.matmul(x8.float(), s.w8.float().t()) * (x_scale * s.w_scale.t()) + s.b.float()
        if s.res is not None:
            y = y + s.res.float()
        return y.to(s.x.dtype)
    if op == "store":
        _write(s.held, s.k, s.v, s.places)
        return [t.to(s.k.dtype) for t in _read(s.held, s.places)]
    out = torch.empty(s.q.shape, dtype=s.q.dtype, device="cuda")
    q0 = k0 = 0
    for i, (new, old) in enumerate(s.lens):
        L = new + old
        if op == "attn":
            k, v = s.k[k0:k0 + L], s.v[k0:k0 + L]
        else:
            j = torch.arange(L, device="cuda")
            k, v = _read(s.held, s.table[i].long()[j // s.page] * s.page + j % s.page)
        out[q0:q0 + new] = _attention(s.q[q0:q0 + new], k, v, case["dim"] ** -0.5).to(s.q.dtype)
        q0, k0 = q0 + new, k0 + L
    return out


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    if not s.own:
        return _plain(s)
    import paper_2501_09253_amd as ps
    op = s.case["op"]
    if op == "linear":
        return s.layer.forward(s.x, res=s.res, y=s.y)
    if op == "store":
        s.store.write(s.k, s.v, s.places)
        return list(s.store.read(s.places, ps.BF16 if s.case["dtype"] == "bf16" else ps.F32))
    if op == "attn":
        return ps.prompt_attention(s.q, s.k, s.v, s.cu_q, s.cu_k, max_q=s.max_q, max_k=s.max_k)
    return s.store.attention(s.q, s.cu_q, s.key_len, s.table, s.page, max_q=s.max_q, max_k=s.max_k)


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    op = case["op"]
    if op == "linear":
        rows, K, N = case["rows"], case["K"], case["N"]
        return {"bytes": rows * K * size + K * N + rows * N * size * (2 if case["res"] else 1) + 4 * N + N * size,
                "flops": 2 * rows * K * N}
    Hk, D = case["kv_heads"], case["dim"]
    if op == "store":
        values = 2 * case["tokens"] * Hk * D            # keys and values: read, held in 8 bits, read, returned
        return {"bytes": values * (2 * size + 2) + 2 * (values // D) * 4 + 16 * case["tokens"], "flops": 4 * values}
    lens = _lens(case)
    H = case["heads"]
    new, all_ = sum(n for n, _ in lens), sum(n + o for n, o in lens)
    pairs = sum(n * o + n * (n + 1) // 2 for n, o in lens)
    kv = all_ * Hk * (D * size if op == "attn" else D + 4)
    return {"bytes": 2 * new * H * D * size + 2 * kv, "flops": 4 * pairs * H * D}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _steps64(x):
    """The values that x [..., D] stands for in 8 bits: each the nearest of 255 equal steps between -amax and amax."""
    x = x.double()
    peak = x.abs().max(dim=-1, keepdim=True).values
    return torch.where(peak == 0, x, torch.round(127 * x / peak) * peak / 127)


def exact(case, seed):
    i = _Inputs(case, seed)
    op = case["op"]
    dt = torch.float64
    if op == "linear":
        y = torch.mm(_steps64(i.x), _steps64(i.w.t()).t().contiguous()) + i.b.to(dt)
        return y if i.res is None else y + i.res.to(dt)
    if op == "store":
        return [_steps64(i.k), _steps64(i.v)]
    k, v = (i.k.to(dt), i.v.to(dt)) if op == "attn" else (_steps64(i.k), _steps64(i.v))
    G = case["heads"] // case["kv_heads"]
    out = torch.zeros(i.q.shape, dtype=dt, device="cuda")
    for n in range(len(i.lens)):
        new, L = i.lens[n][0], sum(i.lens[n])
        for h in range(case["heads"]):
            kh = k[i.cu_k[n]:i.cu_k[n + 1], h // G].contiguous()
            vh = v[i.cu_k[n]:i.cu_k[n + 1], h // G].contiguous()
            for a in range(0, new, 4096):
                b = min(new, a + 4096)
                row = slice(i.cu_q[n] + a, i.cu_q[n] + b)
                logit = torch.mm(i.q[row, h].to(dt).contiguous(), kh.t().contiguous()) / math.sqrt(case["dim"])
                allowed = torch.ones((b - a, L), dtype=torch.bool, device="cuda").tril(L - new + a)
                logit = torch.where(allowed, logit, torch.tensor(-math.inf, dtype=dt, device="cuda"))
                out[row, h] = torch.mm(torch.softmax(logit, -1), vh)
    return out
