"""Causal attention over packed prompts (pserve_prompt_attention) against the plain 64-bit form, row by row within the error
bound of its own sums (tests/prompt_oracle.py)."""
import pytest
import torch

import paper_2501_09253_amd as ps
import prompt_oracle as po

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def starts(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def make(seed, shape, dtype, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * gain).to(dtype)


def check(got, q, k, v, lq, lk, causal=True, scale=None, skip=0):
    D, dtype = q.shape[2], q.dtype
    scale = D ** -0.5 if scale is None else scale
    got = got.double().cpu()
    cq, ck = starts(lq), starts(lk)
    for s in range(len(lq)):
        out, bound, size = po.attention(q[cq[s] + skip:cq[s + 1] + skip], k[ck[s]:ck[s + 1]], v[ck[s]:ck[s + 1]], scale, causal)
        tol = po.attention_tolerance(out, bound, size, dtype, D, lk[s])
        err = (got[cq[s] + skip:cq[s + 1] + skip] - out).abs()
        assert torch.all(err <= tol), (s, lq[s], lk[s], (err / tol).max().item())


HEADS = [(4, 4, 64), (8, 2, 128), (3, 1, 80), (2, 1, 16), (6, 2, 32), (5, 5, 96), (40, 2, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
@pytest.mark.parametrize("lens", [[1], [2, 1, 0, 3], [77, 77, 5], [15, 16, 17, 33, 64, 65, 130]])
def test_packed_prompts(lens, heads, kv_heads, dim, dtype):
    T = sum(lens)
    q, k, v = (make(i, (T, h, dim), DT[dtype]) for i, h in ((1, heads), (2, kv_heads), (3, kv_heads)))
    got = ps.prompt_attention(q.cuda(), k.cuda(), v.cuda(), ints(starts(lens)))
    check(got, q, k, v, lens, lens)
    hinted = ps.prompt_attention(q.cuda(), k.cuda(), v.cuda(), ints(starts(lens)), max_q=max(lens), max_k=max(lens))
    check(hinted, q, k, v, lens, lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk", [([1, 1, 1], [1, 300, 64]), ([5, 40, 1, 0], [900, 40, 0, 7]), ([20, 3], [4, 3]), ([1], [2600]),
                                   ([70, 130, 2], [333, 1029, 77])])
def test_keys_of_other_lengths(lq, lk, causal, dtype):
    """More keys than queries (a prompt being extended, single tokens), fewer (rows without a key give zeros), none."""
    H, Hk, D = 8, 2, 64
    q, k, v = make(1, (sum(lq), H, D), DT[dtype]), make(2, (sum(lk), Hk, D), DT[dtype]), make(3, (sum(lk), Hk, D), DT[dtype])
    for hint in (0, max(lk)):
        got = ps.prompt_attention(q.cuda(), k.cuda(), v.cuda(), ints(starts(lq)), ints(starts(lk)), causal=causal, max_k=hint)
        check(got, q, k, v, lq, lk, causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_longer_prompts(dtype):
    lens = [700, 1, 411]
    q, k, v = make(1, (sum(lens), 2, 128), DT[dtype], 2.0), make(2, (sum(lens), 1, 128), DT[dtype], 2.0), make(3, (sum(lens), 1, 128), DT[dtype])
    got = ps.prompt_attention(q.cuda(), k.cuda(), v.cuda(), ints(starts(lens)), scale=0.3)
    check(got, q, k, v, lens, lens, scale=0.3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gain,where", [(60.0, "rising"), (60.0, "falling"), (200.0, "last"), (-60.0, "rising")])
def test_large_scores(gain, where, dtype):
    """Scores of some hundred that rise or fall along the keys: the softmax reference has to follow them."""
    L, H, D = 300, 2, 64
    q, k, v = make(1, (L, H, D), DT[dtype], 0.1), make(2, (L, H, D), DT[dtype], 0.1), make(3, (L, H, D), DT[dtype])
    along = {"rising": torch.linspace(-1, 1, L), "falling": torch.linspace(1, -1, L), "last": (torch.arange(L) % 97 == 96).float()}[where]
    q[:, :, 0] = 8.0
    k[:, :, 0] = (along * gain)[:, None].to(k.dtype)
    got = ps.prompt_attention(q.cuda(), k.cuda(), v.cuda(), ints([0, L]))
    check(got, q, k, v, [L], [L])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(dtype):
    """q, k and v as slices of one projection, heads outside tokens, and an output that is a slice."""
    lens, H, Hk, D = [33, 70, 1], 6, 2, 64
    T = sum(lens)
    cu = ints(starts(lens))
    qkv = make(1, (T, H + 2 * Hk, D), DT[dtype]).cuda()
    q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    want = ps.prompt_attention(q.contiguous(), k.contiguous(), v.contiguous(), cu)
    check(want, q.cpu(), k.cpu(), v.cpu(), lens, lens)
    assert torch.equal(ps.prompt_attention(q, k, v, cu), want)
    swap = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    out = swap(torch.zeros_like(want))
    assert torch.equal(ps.prompt_attention(swap(q), swap(k), swap(v), cu, out=out), want) and not out.is_contiguous()
    wide = torch.full((T, H, D + 16), 7.0, dtype=DT[dtype], device="cuda")
    ps.prompt_attention(q, k, v, cu, out=wide[:, :, :D])
    assert torch.equal(wide[:, :, :D], want) and torch.all(wide[:, :, D:] == 7.0)
    one = k[:, :1].expand(T, Hk, D)                                     # one key head shown as two
    assert torch.equal(ps.prompt_attention(q, one, v, cu), ps.prompt_attention(q, one.contiguous(), v, cu))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_rows_outside_the_sequences_and_what_no_query_sees(dim, dtype):
    """Rows of no sequence stay as they were; infinities and NaN behind a query, in other sequences and between them do not
    reach it; a value that is not finite reaches the queries that see it."""
    H, Hk = 4, 2
    lens, lead, tail = [50, 37, 100], 3, 9
    T = lead + sum(lens) + tail
    cu = ints([lead + c for c in starts(lens)])
    q, k, v = make(1, (T, H, dim), DT[dtype]), make(2, (T, Hk, dim), DT[dtype]), make(3, (T, Hk, dim), DT[dtype])
    out = torch.full((T, H, dim), 5.0, dtype=DT[dtype], device="cuda")
    want = ps.prompt_attention(q.cuda(), k.cuda(), v.cuda(), cu, out=out.clone())
    check(want, q, k[lead:], v[lead:], lens, lens, skip=lead)
    assert torch.all(want[:lead] == 5.0) and torch.all(want[T - tail:] == 5.0)
    at = lead + 50 + 20                                                 # token 20 of the second sequence
    for bad in (float("inf"), float("-inf"), float("nan")):
        for t in (k, v):
            x = t.clone()
            x[:lead], x[T - tail:] = bad, bad
            args = [a.cuda() for a in ((q, x, v) if t is k else (q, k, x))]
            assert torch.equal(ps.prompt_attention(*args, cu, out=out.clone()), want)
            x[at, :, 5] = bad
            args = [a.cuda() for a in ((q, x, v) if t is k else (q, k, x))]
            got = ps.prompt_attention(*args, cu, out=out.clone())
            inside = slice(at, lead + 87)
            assert torch.equal(got[:at], want[:at]) and torch.equal(got[lead + 87:], want[lead + 87:])
            if t is v:
                assert not torch.isfinite(got[inside, :, 5]).any()
                rest = [d for d in range(dim) if d != 5]
                assert torch.equal(got[inside][:, :, rest], want[inside][:, :, rest])


def test_sequence_numbers_beyond_a_wavefront():
    """More sequences than lanes look for them, many of them empty."""
    lens = [(7 * i) % 5 if i % 3 else 0 for i in range(300)]
    q, k, v = make(1, (sum(lens), 2, 64), DT["bf16"]), make(2, (sum(lens), 2, 64), DT["bf16"]), make(3, (sum(lens), 2, 64), DT["bf16"])
    got = ps.prompt_attention(q.cuda(), k.cuda(), v.cuda(), ints(starts(lens)))
    check(got, q, k, v, lens, lens)


def test_starts_that_point_outside_are_cut():
    """Starts beyond the tensors or below zero: what lies inside is computed, nothing else is touched."""
    q, k, v = (make(i, (40, 2, 64), DT["bf16"]) for i in (1, 2, 3))
    got = ps.prompt_attention(q.cuda(), k.cuda(), v.cuda(), ints([-5, 25, 90]))
    check(got, q, k, v, [25, 15], [25, 15])


def test_graph_and_other_streams():
    """Captured and replayed on changed inputs between eager calls; a call on a side stream."""
    lens = [90, 33, 260]
    cu = ints(starts(lens))
    q, k, v = (make(i, (sum(lens), h, 128), DT["bf16"]).cuda() for i, h in ((1, 8), (2, 2), (3, 2)))
    one_q, one_cu = q[:3].clone(), ints([0, 1, 2, 3])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call = lambda: (ps.prompt_attention(q, k, v, cu), ps.prompt_attention(one_q, k, v, one_cu, cu, max_q=1, max_k=2600))
    with torch.cuda.stream(side):
        want = call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for i in range(4):
        q.copy_(make(10 + i, q.shape, q.dtype))
        one_q.copy_(q[5:8])
        graph.replay()
        torch.cuda.synchronize()
        again = call()
        assert all(torch.equal(a, b) for a, b in zip(got, again))
    assert not torch.equal(got[0], want[0])
