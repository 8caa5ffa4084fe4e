"""What the 8-bit store gives back, bit for bit, and the places that it has."""
import pytest
import torch

import paper_2501_09253_amd as ps
import prompt_exact as pe
import prompt_oracle as po
from test_gpu_prompt_attention import ints, make

pytestmark = pytest.mark.gpu


def nearest_bf16(x):
    """64-bit numbers in bf16's normal range to the nearest of bf16, halves to even, without a step between."""
    assert torch.all((x == 0) | (x.abs() >= 2.0 ** -126))
    u = x.view(torch.int64)
    u = (u + (1 << 44) - 1 + ((u >> 45) & 1)) & ~((1 << 45) - 1)       # 53 bits to 8; the sign is a bit of its own
    return u.view(torch.float64)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,dim", [(8, 128), (12, 64), (3, 80)])
def test_values_are_rounded_once(heads, dim, dtype):
    """Whole number times fp32 scale has up to 31 bits: of the fp32 rows 3 to 55 values lie so close to the middle of two bf16 numbers that
    their fp32 product is the middle."""
    rows = 4000
    k, v = make(1, (rows, heads, dim), dtype), make(2, (rows, heads, dim), dtype, 30.0)
    store, at = ps.KV8(rows, heads, dim), torch.arange(rows, device="cuda")
    store.write(k.cuda(), v.cuda(), at)
    for x, half, whole in zip((k, v), store.read(at, ps.BF16), store.read(at, ps.F32)):
        q, s = po.steps(x)
        exact = q * s.float().double()                                  # 31 bits: exact in 64
        near = nearest_bf16(exact)
        assert (near != exact.float().bfloat16().double()).sum() >= (3 if dtype == torch.float32 else 0)
        assert torch.equal(half.cpu().double(), near)
        assert torch.equal(whole.cpu(), exact.float())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new", [1, 90])
@pytest.mark.parametrize("places,page", [(100, 16), (1000, 64), (1000, 1024), (700, 512), (33, 32)])
def test_places_of_a_partly_filled_last_page(places, page, new, dtype):
    """A store whose places are no multiple of the page: keys on its last page count up to the last place, those behind it do not."""
    H, Hk, D = 4, 2, 64
    pages = -(-places // page)
    k, v = make(2, (places, Hk, D), dtype), make(3, (places, Hk, D), dtype)
    store = ps.KV8(places, Hk, D)
    store.write(k.cuda(), v.cuda(), torch.arange(places, device="cuda"))
    order = [pages - 1] + list(range(pages - 1))                       # the partly filled page first: its missing keys lie in the middle
    key = [p * page + j for p in order for j in range(page)]
    length = min(len(key), places + 5)
    here = [j for j in key[:length] if j < places]
    q = make(1, (new, H, D), dtype)
    for hint in (0, length):
        got = store.attention(q.cuda(), ints([0, new]), ints([length]), ints([order]), page, causal=False, max_q=new, max_k=hint).double()
        out, bound, _, size = pe.attention(q, po.held(k[here]), po.held(v[here]), D ** -0.5, False)
        tol = pe.tolerance(out, bound, size, dtype, D, len(here), pe.ONE_PIECE, scales=4)
        assert torch.all((got.cpu() - out).abs() <= tol), ((got.cpu() - out).abs() / tol).max()
    far = store.attention(q.cuda(), ints([0, new]), ints([page]), ints([[pages]]), page, causal=False)
    assert torch.all(far == 0)                                          # a page behind the last


def test_captured_writes_of_many_rows():
    """Replayed with other rows and places, some twice and some outside, between eager writes of the same store."""
    rows, places, heads, dim = 700, 400, 3, 64
    k, v = make(1, (rows, heads, dim), torch.bfloat16).cuda(), make(2, (rows, heads, dim), torch.bfloat16).cuda()
    at = torch.zeros(rows, dtype=torch.int64, device="cuda")
    store, plain = ps.KV8(places, heads, dim), ps.KV8(places, heads, dim)
    every = torch.arange(places, device="cuda")
    store.write(k, v, at)
    plain.write(k, v, at)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        store.write(k, v, at)
    for i in range(6):
        k.copy_(make(10 + i, k.shape, k.dtype))
        v.copy_(make(20 + i, v.shape, v.dtype))
        at.copy_(torch.randint(-20, places + 20, (rows,), generator=torch.Generator().manual_seed(i)))
        graph.replay() if i % 3 else store.write(k, v, at)
        last = {p: j for j, p in enumerate(at.tolist()) if 0 <= p < places}
        rest = sorted(last.values())                                    # the rows that count, each place once
        plain.write(k[rest], v[rest], at[rest])
        assert all(torch.equal(a, b) for a, b in zip(store.read(every, ps.F32), plain.read(every, ps.F32)))
