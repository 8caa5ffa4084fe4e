"""Scores that are not finite in the prompt attention, whatever the head size and the kernel: +infinity and NaN make the row NaN, -infinity
weighs nothing."""
import pytest
import torch

import paper_2501_09253_amd as ps
import prompt_exact as pe
import prompt_oracle as po
from test_gpu_kv8 import paged
from test_gpu_prompt_attention import ints, make, starts

pytestmark = pytest.mark.gpu

# queries, keys, heads, key/value heads: tiles of 16 rows (whole, and their keys cut), of 128, of 128 in shares, of 256
CALLS = {"16 rows": (5, 60, 4, 2), "16 rows, cut": (2, 1500, 6, 2), "128 rows": (77, 77, 160, 160), "128 rows, shares": (90, 1300, 4, 2),
         "256 rows": (1100, 1100, 64, 8)}


def run(q, k, v, scale=None, causal=True):
    """(got, wanted, tolerance), one sequence."""
    (Lq, _, D), Lk = q.shape, k.shape[0]
    scale = D ** -0.5 if scale is None else scale
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    got = ps.prompt_attention(q, k, v, ints([0, Lq]), ints([0, Lk]), causal=causal, scale=scale, max_q=Lq, max_k=Lk)
    out, bound, _, size = pe.attention(q, k, v, scale, causal)
    return got.double(), out, pe.tolerance(out, bound, size, q.dtype, D, Lk, pe.ONE_PIECE)


def same(got, out, tol):
    assert torch.equal(got.isnan(), out.isnan()), (got.isnan().sum().item(), out.isnan().sum().item())
    err = (got - out).abs()
    assert torch.all((err <= tol) | out.isnan()), (err / tol).nan_to_num().max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("dim", range(16, 129, 16))
def test_infinite_keys_at_every_head_size(dim, call, dtype):
    """A key with an infinity in its first values, in the middle and in its last: rows whose query is negative there do not count it, rows
    whose query is positive there are NaN."""
    Lq, Lk, H, Hk = CALLS[call]
    q, k, v = make(1, (Lq, H, dim), dtype), make(2, (Lk, Hk, dim), dtype), make(3, (Lk, Hk, dim), dtype)
    for at, channel, sign in ((Lk - Lq, 0, 1.0), (Lk - Lq + Lq // 3, 7, -1.0), (Lk - Lq + Lq // 2, dim // 2, 1.0), (0, dim - 1, -1.0), (3, 3, 1.0)):
        kk, qq = k.clone(), q.clone()
        kk[at, :, channel] = sign * float("inf")
        same(*run(qq, kk, v))                                           # queries of either sign
        qq[:, :, channel] = -sign * (qq[:, :, channel].abs() + 0.125)
        got, out, tol = run(qq, kk, v)                                  # all of them with a score of -infinity
        assert not out.isnan().any()
        same(got, out, tol)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim", range(16, 129, 16))
def test_rows_with_no_other_score_are_zero(dim, dtype):
    """The first token sees one key, of score -infinity; a call in which all scores are -infinity."""
    for Lq, Lk, H, Hk in CALLS.values():
        q, k, v = make(1, (Lq, H, dim), dtype), make(2, (Lk, Hk, dim), dtype), make(3, (Lk, Hk, dim), dtype)
        q[:, :, 2] = -1.0
        kk = k.clone()
        kk[:Lk - Lq + 1, :, 2] = float("inf")
        got, out, tol = run(q, kk, v)
        assert torch.all(got[0] == 0) and torch.all(out[0] == 0)
        same(got, out, tol)
        kk[:, :, 2] = float("inf")
        assert torch.all(run(q, kk, v)[0] == 0)


@pytest.mark.parametrize("dim", [32, 80, 128])
def test_packed_neighbours_with_infinite_keys(dim):
    """Sequences side by side: a key of one of them has no part in the others."""
    lens, H, Hk = [70, 3, 130], 6, 2
    q, k, v = (make(i, (sum(lens), h, dim), torch.bfloat16).cuda() for i, h in ((1, H), (2, Hk), (3, Hk)))
    q[:, :, 1] = -1.0
    k[::11, :, 1] = float("inf")
    got, at = ps.prompt_attention(q, k, v, ints(starts(lens))).double(), starts(lens)
    for s, L in enumerate(lens):
        r = slice(at[s], at[s + 1])
        out, bound, _, size = pe.attention(q[r], k[r], v[r], dim ** -0.5)
        same(got[r], out, pe.tolerance(out, bound, size, q.dtype, dim, L, pe.ONE_PIECE))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("dim", [64, 80, 128])
def test_scores_that_overflow_with_their_scale(dim, call, dtype):
    """q.k in the range of fp32, the scale times it not: the score counts as infinite, +: the row is NaN, -: the key weighs nothing."""
    Lq, Lk, H, Hk = CALLS[call]
    q, k, v = make(1, (Lq, H, dim), dtype, 0.2), make(2, (Lk, Hk, dim), dtype, 0.2), make(3, (Lk, Hk, dim), dtype)
    q[:, :, 0], k[:, :, 0] = 2.0 ** 60, 0.0
    for at in (3, Lk - Lq + Lq // 2):
        for sign in (1.0, -1.0):
            big, inf = k.clone(), k.clone()
            big[at, :, 0], inf[at, :, 0] = sign * 2.0 ** 65, sign * float("inf")    # 2^125 times 8 log2(e): beyond 2^128
            got = run(q, big, v, scale=8.0)[0]
            _, out, tol = run(q, inf, v, scale=8.0)
            assert out.isnan().any() == (sign > 0)
            same(got, out, tol)
            table, places, total = paged([Lk], 64, 4)
            store = ps.KV8(total, Hk, dim)
            store.write(big.cuda(), v.cuda(), places)
            got = store.attention(q.cuda(), ints([0, Lq]), ints([Lk]), table, 64, scale=8.0, max_q=Lq, max_k=Lk).double()
            inf = po.held(k)
            inf[at], inf[at, :, 0] = 0.0, sign * float("inf")
            out, bound, _, size = pe.attention(q.cuda(), inf.cuda(), po.held(v).cuda(), 8.0)
            same(got, out, pe.tolerance(out, bound, size, dtype, dim, Lk, pe.ONE_PIECE, scales=4))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -112, -2.0 ** -112])
def test_small_scales_of_large_products(scale, call, dtype):
    """q.k of about 2^114: all keys weigh the same where the scale is 0, and what the formula says where it is small."""
    Lq, Lk, H, Hk = CALLS[call]
    q, k, v = make(1, (Lq, H, 64), dtype), make(2, (Lk, Hk, 64), dtype), make(3, (Lk, Hk, 64), dtype)
    same(*run(q * 2.0 ** 55, k * 2.0 ** 56, v, scale=scale))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("call", list(CALLS))
def test_large_keys_of_the_store_with_a_large_scale(call, dtype):
    """A key's 8-bit scale times the scores' leaves fp32's range, the key's score does not: it is 0."""
    Lq, Lk, H, Hk = CALLS[call]
    q, k, v = make(1, (Lq, H, 64), dtype, 0.02), make(2, (Lk, Hk, 64), dtype, 0.02), make(3, (Lk, Hk, 64), dtype)
    q[:, :, 0] = 0.0
    k[Lk - Lq:, :, 0] = 2.0 ** 127
    table, places, total = paged([Lk], 64, 4)
    store = ps.KV8(total, Hk, 64)
    store.write(k.cuda(), v.cuda(), places)
    got = store.attention(q.cuda(), ints([0, Lq]), ints([Lk]), table, 64, scale=1000.0, max_q=Lq, max_k=Lk).double()
    kk = po.held(k)
    kk[:, :, 0] = 0.0
    out, bound, _, size = pe.attention(q.cuda(), kk.cuda(), po.held(v).cuda(), 1000.0)
    same(got, out, pe.tolerance(out, bound, size, dtype, 64, Lk, pe.ONE_PIECE, scales=4))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("dim", [16, 64, 80, 128])
def test_queries_that_are_not_finite(dim, call, dtype):
    """NaN and infinities in some queries reach their own rows only: all keys of one sign against an infinite query give NaN or zeros."""
    Lq, Lk, H, Hk = CALLS[call]
    q, k, v = make(1, (Lq, H, dim), dtype), make(2, (Lk, Hk, dim), dtype), make(3, (Lk, Hk, dim), dtype)
    k[:, :, 1] = k[:, :, 1].abs() + 0.125
    bad = q.clone()
    bad[Lq // 2, ::2, 1], bad[Lq // 2, 1::2, 1], bad[Lq - 1, :, dim - 1] = float("inf"), float("-inf"), float("nan")
    finite = [i for i in range(Lq) if i not in (Lq // 2, Lq - 1)]
    got, _, _ = run(bad, k, v)
    _, out, tol = run(q, k, v)
    assert torch.all((got - out).abs()[finite] <= tol[finite])
    if Lq // 2 != Lq - 1:
        assert got[Lq // 2, ::2].isnan().all() and torch.all(got[Lq // 2, 1::2] == 0)
    assert got[Lq - 1].isnan().all()
