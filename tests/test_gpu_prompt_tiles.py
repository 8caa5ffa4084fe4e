"""The prompt attention on calls large enough for its wide tiles and for shares of the keys, against the plain 64-bit form on the
GPU; what the tiles' fast loop assumes of the scores, and does not get."""
import pytest
import torch

import paper_2501_09253_amd as ps
import prompt_oracle as po
from test_gpu_prompt_attention import DT, ints, make, starts
from test_gpu_kv8 import paged

pytestmark = pytest.mark.gpu


def near(got, q, k, v, lq, lk, causal=True, scale=None, extra=0.0):
    D, cq, ck = q.shape[2], starts(lq), starts(lk)
    for s in range(len(lq)):
        if lq[s] == 0:
            continue
        out, bound, size = po.attention_by_heads(q[cq[s]:cq[s + 1]], k[ck[s]:ck[s + 1]], v[ck[s]:ck[s + 1]], D ** -0.5 if scale is None else scale, causal)
        tol = po.attention_tolerance(out, bound, size, q.dtype, D, lk[s]) + extra * po.U * bound
        err = (got[cq[s]:cq[s + 1]].double() - out).abs()
        assert torch.all(err <= tol), (s, lq[s], lk[s], (err / tol).max().item())


SIZES = [([300] * 40, None, 16, 16, 64), ([257, 1, 700, 64, 513, 0, 2048, 77] * 3, None, 16, 4, 128), ([1500], None, 24, 8, 96),
         ([130, 260], [3000, 4100], 8, 2, 128), ([512, 300], [2048, 2048], 12, 12, 64), ([2100], [700], 32, 8, 128), ([40], [9000], 16, 2, 64)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk,heads,kv_heads,dim", SIZES)
def test_large_calls(lq, lk, heads, kv_heads, dim, causal):
    lk = lq if lk is None else lk
    q, k, v = (make(i, (sum(n), h, dim), DT["bf16"]).cuda() for i, n, h in ((1, lq, heads), (2, lk, kv_heads), (3, lk, kv_heads)))
    got = ps.prompt_attention(q, k, v, ints(starts(lq)), ints(starts(lk)), causal=causal, max_q=max(lq), max_k=max(lk))
    near(got, q, k, v, lq, lk, causal)


@pytest.mark.parametrize("lq,lk,heads,kv_heads,dim", SIZES[1:])
def test_large_calls_over_the_store(lq, lk, heads, kv_heads, dim):
    lk = lq if lk is None else lk
    q, k, v = (make(i, (sum(n), h, dim), DT["bf16"]).cuda() for i, n, h in ((1, lq, heads), (2, lk, kv_heads), (3, lk, kv_heads)))
    table, places, total = paged(lk, 32, 4)
    store = ps.KV8(total, kv_heads, dim)
    store.write(k, v, places)
    got = store.attention(q, ints(starts(lq)), ints(lk), table, 32, max_q=max(lq), max_k=max(lk))
    near(got, q, po.held(k), po.held(v), lq, lk, extra=4)


@pytest.mark.parametrize("dim,heads", [(64, 64), (128, 64)])
@pytest.mark.parametrize("kind", ["rising", "falling", "late peak", "negative scale", "zero scale", "huge values"])
def test_scores_that_leave_the_first_reference(kind, dim, heads):
    """The tiles' fast loop takes the first 32 scores of a row as its reference; scores far above it, and values near the largest number,
    have to come out all the same."""
    L = 2100
    q, k, v = make(1, (L, heads, dim), torch.bfloat16, 0.1), make(2, (L, 1, dim), torch.bfloat16, 0.1), make(3, (L, 1, dim), torch.bfloat16)
    scale = dim ** -0.5
    q[:, :, 0] = 8.0
    step = torch.linspace(-1, 1, L)
    if kind == "rising":
        k[:, 0, 0] = (400 * step).bfloat16()
    elif kind == "falling":
        k[:, 0, 0] = (-400 * step).bfloat16()
    elif kind == "late peak":
        k[1333, 0, 0] = 600.0
    elif kind == "negative scale":
        k[:, 0, 0] = (-300 * step).bfloat16()
        scale = -scale
    elif kind == "zero scale":
        scale = 0.0
    else:
        k[:, 0, 0] = (20 * step).bfloat16()
        v = (v.float() * 2.0 ** 120).bfloat16()
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    got = ps.prompt_attention(q, k, v, ints([0, L]), scale=scale, max_q=L, max_k=L)
    near(got, q, k, v, [L], [L], scale=scale)


def test_what_is_not_finite_far_behind_the_diagonal():
    """NaN and infinities in values and keys that only the later rows of a wide tile see."""
    L, H, D = 2048, 64, 128
    q, k, v = make(1, (L, H, D), torch.bfloat16).cuda(), make(2, (L, 8, D), torch.bfloat16).cuda(), make(3, (L, 8, D), torch.bfloat16).cuda()
    cu = ints([0, L])
    want = ps.prompt_attention(q, k, v, cu, max_q=L, max_k=L)
    for at in (40, 1000, 1030, 2047):
        for bad in (float("nan"), float("inf"), float("-inf")):
            for side in (0, 1):
                kv = [k.clone(), v.clone()]
                kv[side][at, 3, 17] = bad
                got = ps.prompt_attention(q, *kv, cu, max_q=L, max_k=L)
                others = [h for h in range(H) if h // 8 != 3]
                assert torch.equal(got[:at], want[:at]) and torch.equal(got[:, others], want[:, others])
                if side:
                    assert not torch.isfinite(got[at:, 24:32, 17]).any()
                elif bad != bad:
                    assert torch.isnan(got[at:, 24:32]).all()
