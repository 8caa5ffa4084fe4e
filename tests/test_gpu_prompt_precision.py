"""How exact the prompt attention is on each of its paths, and that every key counts once: bounds that a key left out, a key counted twice, or a
weight rounded to one bf16 number where two are promised does not meet (tests/test_prompt_bounds.py plants these)."""
import pytest
import torch

import paper_2501_09253_amd as ps
import prompt_exact as pe
import prompt_oracle as po
from test_gpu_kv8 import paged
from test_gpu_prompt_attention import ints, make, starts

pytestmark = pytest.mark.gpu

# queries, keys, heads, key/value heads, values of a head; packed bf16 in tiles of 256 rows?
SHORT = [([100, 7, 77], [100, 7, 77], 4, 2, 64, False), ([77] * 4, [77] * 4, 80, 40, 64, False), ([77] * 5, [77] * 5, 40, 40, 80, False), ([1] * 6, [300, 1, 77, 129, 8, 250], 8, 2, 128, False),
         ([120, 33], [300, 250], 64, 16, 128, False)]
LONG = [([1, 2, 1], [3000, 513, 1290], 8, 2, 128, False), ([40], [9000], 16, 2, 64, False), ([130, 260], [3000, 4100], 8, 2, 128, False), ([700, 1, 411], [700, 1, 411], 20, 20, 96, False),
        ([512], [4096], 32, 8, 64, True), ([2100], [2100], 32, 8, 128, True), ([1500, 257], [1500, 900], 48, 4, 64, True)]


def run(q, k, v, lq, lk, causal, stored):
    if not stored:
        return ps.prompt_attention(q, k, v, ints(starts(lq)), ints(starts(lk)), causal=causal, max_q=max(lq), max_k=max(lk))
    table, places, total = paged(lk, 32, 4)
    store = ps.KV8(total, k.shape[1], k.shape[2])
    store.write(k, v, places)
    return store.attention(q, ints(starts(lq)), ints(lk), table, 32, causal=causal, max_q=max(lq), max_k=max(lk))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("stored", [False, True])
@pytest.mark.parametrize("lq,lk,heads,kv_heads,dim,wide", SHORT + LONG)
def test_error_of_each_path(lq, lk, heads, kv_heads, dim, wide, stored, causal, dtype):
    q, k, v = (make(i, (sum(n), h, dim), dtype).cuda() for i, n, h in ((1, lq, heads), (2, lk, kv_heads), (3, lk, kv_heads)))
    got = run(q, k, v, lq, lk, causal, stored)
    assert torch.equal(got, run(q, k, v, lq, lk, causal, stored))       # the same sums in the same order
    if stored:
        k, v = po.held(k), po.held(v)
    piece = pe.ONE_PIECE if wide and not stored else pe.TWO_PIECES
    cq, ck = starts(lq), starts(lk)
    for s in range(len(lq)):
        out, bound, spread, size = pe.attention(q[cq[s]:cq[s + 1]], k[ck[s]:ck[s + 1]], v[ck[s]:ck[s + 1]], dim ** -0.5, causal)
        err = got[cq[s]:cq[s + 1]].double() - out
        tol = pe.tolerance(out, bound, size, dtype, dim, lk[s], piece, scales=4 if stored else 0)
        assert torch.all(err.abs() <= tol), (s, (err.abs() / tol).max().item())
        most = pe.norm_bound(out, bound, spread, size, dtype, dim, lk[s], piece)
        assert err.norm() <= most, (s, (err.norm() / out.norm()).item(), (most / out.norm()).item())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("stored", [False, True])
@pytest.mark.parametrize("lq,lk,heads,kv_heads,dim", [c[:5] for c in SHORT + LONG] + [([1] * 9, [1, 127, 128, 129, 511, 512, 513, 640, 4097], 8, 2, 128),
                                                      ([90] * 5, [90, 512, 575, 1344, 2049], 8, 2, 64), ([300] * 3, [1025, 1984, 3001], 32, 8, 64)])
def test_every_key_counts_once(lq, lk, heads, kv_heads, dim, stored, dtype):
    """All scores alike, key j has a 1 in channel j % dim: a row that sees n keys gives the shares of n that fall to each channel."""
    q = torch.zeros(sum(lq), heads, dim, dtype=dtype, device="cuda")
    k = make(2, (sum(lk), kv_heads, dim), dtype).cuda()
    j = torch.cat([torch.arange(n) for n in lk]).cuda()
    v = (j[:, None] % dim == torch.arange(dim, device="cuda")).to(dtype)[:, None].expand(-1, kv_heads, dim).contiguous()
    channel = torch.arange(dim, device="cuda")
    for causal in (True, False):
        got, cq = run(q, k, v, lq, lk, causal, stored).double(), starts(lq)
        for s in range(len(lq)):
            n = torch.full((lq[s],), lk[s], device="cuda")
            if causal:
                n = (torch.arange(lq[s], device="cuda") + lk[s] - lq[s] + 1).clamp(0, lk[s])
            share = ((n[:, None] - channel + dim - 1) // dim).clamp(min=0) / n[:, None].clamp(min=1).double()
            # weights of 1 are exact; the sum of the weights, its reciprocal and the product in fp32, a value's scale, the result's rounding
            tol = ((2 * lk[s] + 8) * po.U + po.HALF[dtype]) * share
            assert torch.all((got[cq[s]:cq[s + 1]] - share[:, None]).abs() <= tol[:, None]), (s, causal)
