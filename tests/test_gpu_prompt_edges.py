"""Calls of the prompt-side operators at the edges of what their documentation allows, and what the binding refuses."""
import pytest
import torch

import paper_2501_09253_amd as ps
import prompt_oracle as po
from test_gpu_kv8 import check_cached, paged, same
from test_gpu_prompt_attention import check, ints, make, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("L", [1, 40])
def test_strides_of_dimensions_of_one(L, dtype):
    """One token or one head: the stride there is any number, an odd one or one past 2^24."""
    D, odd = 64, (1 << 25) + 3
    q, k, v = (make(i, (L, 1, D), dtype) for i in (1, 2, 3))
    show = lambda t: t.as_strided((L, 1, D), (odd if L == 1 else D, odd, 1))
    want = ps.prompt_attention(q.cuda(), k.cuda(), v.cuda(), ints([0, L]))
    check(want, q, k, v, [L], [L])
    out = torch.empty_like(want)
    assert torch.equal(ps.prompt_attention(show(q.cuda()), show(k.cuda()), show(v.cuda()), ints([0, L]), out=show(out)), want)
    store, at = ps.KV8(64, 1, D), torch.arange(L, device="cuda")
    store.write(show(k.cuda()), show(v.cuda()), at)
    back = store.read(at, ps.F32)
    same(back[0], po.held(k), torch.float32)
    same(back[1], po.held(v), torch.float32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim", range(16, 129, 16))
def test_every_head_size(dim, dtype):
    """Short prompts and a few tokens over many keys; what lies behind a head in memory is NaN."""
    lq, lk, H, Hk = [5, 40, 3], [5, 40, 1500], 6, 2
    wide = lambda seed, n, h: torch.cat([make(seed, (n, h, dim), dtype), torch.full((n, h, 16), float("nan"), dtype=dtype)], 2)
    q, k, v = wide(1, sum(lq), H), wide(2, sum(lk), Hk), wide(3, sum(lk), Hk)
    cut = lambda t: t[:, :, :dim]
    for hint in (40, 1500):
        got = ps.prompt_attention(cut(q.cuda()), cut(k.cuda()), cut(v.cuda()), ints(starts(lq)), ints(starts(lk)), max_q=40, max_k=hint)
        check(got, cut(q), cut(k), cut(v), lq, lk)


def test_outputs_whose_rows_overlap_are_refused():
    T, H, D = 6, 3, 64
    q = make(1, (T, H, D), torch.bfloat16).cuda()
    cu, room = ints([0, T]), torch.zeros(4 * T * H * D, dtype=torch.bfloat16, device="cuda")
    for strides in ((D, D, 1), (2 * D, D, 1), (H * D, 0, 1), (0, D, 1), (D, (T - 1) * D, 1)):
        with pytest.raises(ps.PserveError, match="overlap"):
            ps.prompt_attention(q, q, q, cu, out=room.as_strided((T, H, D), strides))
    want = ps.prompt_attention(q, q, q, cu)
    for strides in ((H * D, D, 1), (D, T * D, 1), (2 * H * D, D, 1), (D + 16, T * (D + 16), 1)):
        assert torch.equal(ps.prompt_attention(q, q, q, cu, out=room.as_strided((T, H, D), strides)), want)
    with pytest.raises(ps.PserveError, match="overlap"):
        ps.prompt_attention(q, q, q, cu, out=q)


def test_no_tokens_no_keys_no_pages():
    H, D = 4, 64
    none, q = torch.empty(0, H, D, dtype=torch.bfloat16, device="cuda"), make(1, (3, H, D), torch.bfloat16).cuda()
    assert ps.prompt_attention(none, none, none, ints([0, 0])).shape == (0, H, D)
    assert torch.all(ps.prompt_attention(q, none, none, ints([0, 3]), ints([0, 0])) == 0)
    store, empty = ps.KV8(32, H, D), torch.empty(0, dtype=torch.int64, device="cuda")
    store.write(none, none, empty)
    assert store.read(empty, ps.BF16)[0].shape == (0, H, D)
    nothing = torch.empty(1, 0, dtype=torch.int32, device="cuda")
    assert torch.all(store.attention(q, ints([0, 3]), ints([5]), nothing, 16) == 0)
    assert torch.all(store.attention(q, ints([0, 3]), ints([5]), ints([[0]]), 64) == 0)         # a page larger than the store
    layer = ps.Linear8(make(2, (D, 8), torch.bfloat16).cuda(), None, ps.BF16)
    assert layer.forward(none[:, 0]).shape == (0, 8)


def test_two_graphs_and_two_streams_share_nothing():
    """Two captured calls that need workspaces, replayed in turn and beside eager calls on another stream."""
    H, Hk, D = 8, 2, 64
    sets = []
    for seed, (lq, lk) in ((1, ([1, 1], [3000, 40])), (2, ([90], [2500]))):
        q, k, v = make(seed, (sum(lq), H, D), torch.bfloat16), make(seed + 5, (sum(lk), Hk, D), torch.bfloat16), make(seed + 9, (sum(lk), Hk, D), torch.bfloat16)
        args = [t.cuda() for t in (q, k, v)] + [ints(starts(lq)), ints(starts(lk))]
        sets.append((args, dict(max_q=max(lq), max_k=max(lk)), (q, k, v, lq, lk)))
    call = lambda i: ps.prompt_attention(*sets[i][0], **sets[i][1])
    want = [call(0), call(1)]
    for w, (_, _, plain) in zip(want, sets):
        check(w, *plain)
    graphs, outs = [], []
    for i in (0, 1):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(call(i))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for n in range(4):
        for o in outs:
            o.fill_(7)
        graphs[n % 2].replay()
        with torch.cuda.stream(side):
            beside = [call(1 - n % 2) for _ in range(3)]
        graphs[1 - n % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want)) and all(torch.equal(b, want[1 - n % 2]) for b in beside)


@pytest.mark.parametrize("dim", [64, 128])
def test_more_sequences_than_lanes_in_wide_tiles(dim):
    """Prompts and extended prompts, some without tokens or keys, in tiles of many rows whose keys are shared out; packed and stored."""
    n, H, Hk, page = 70, 8, 1, 64
    lq = [(5 * i) % 23 if i % 7 else 0 for i in range(n)]
    lq[40] = 90
    lk = [0 if i % 11 == 5 else lq[i] + (13 * i) % 50 for i in range(n)]
    lk[40], lk[69] = 2300, 1900
    q, k, v = make(1, (sum(lq), H, dim), torch.bfloat16), make(2, (sum(lk), Hk, dim), torch.bfloat16), make(3, (sum(lk), Hk, dim), torch.bfloat16)
    table, places, total = paged(lk, page, 4)
    store = ps.KV8(total, Hk, dim)
    store.write(k.cuda(), v.cuda(), places)
    cu = ints(starts(lq))
    for causal in (True, False):
        for hint in (0, 2300, 1 << 20):
            check(ps.prompt_attention(q.cuda(), k.cuda(), v.cuda(), cu, ints(starts(lk)), causal=causal, max_q=90, max_k=hint), q, k, v, lq, lk, causal)
            check_cached(store.attention(q.cuda(), cu, ints(lk), table, page, causal=causal, max_q=90, max_k=hint), q, k, v, lq, lk, causal)


@pytest.mark.parametrize("heads,dim,dtype", [(40, 128, torch.bfloat16), (300, 16, torch.float32)])
def test_rows_of_many_heads(heads, dim, dtype):
    """More groups in a row than a block takes in one go, places taken twice and left out."""
    rows, total = 200, 150
    k, v = make(1, (rows, heads, dim), dtype), make(2, (rows, heads, dim), dtype)
    places = torch.randint(-3, total, (rows,), generator=torch.Generator().manual_seed(3))
    store = ps.KV8(total, heads, dim)
    for _ in range(2):
        store.write(k.cuda(), v.cuda(), places.cuda())
        last = {p: i for i, p in enumerate(places.tolist()) if p >= 0}
        at = sorted(last)
        got = store.read(torch.tensor(at, device="cuda"), ps.F32)
        same(got[0], po.held(k[[last[p] for p in at]]), torch.float32)
        same(got[1], po.held(v[[last[p] for p in at]]), torch.float32)
        k, v, places = v, k, places.flip(0)


def test_thousands_of_short_sequences():
    """More sequences than a block looks at in one go, single tokens and short prompts, each over its own keys."""
    n, H, Hk, D, page = 5000, 4, 2, 64, 16
    lk = [1 + (7 * i) % 30 for i in range(n)]
    q, k, v = make(1, (n, H, D), torch.bfloat16), make(2, (sum(lk), Hk, D), torch.bfloat16), make(3, (sum(lk), Hk, D), torch.bfloat16)
    some = [0, 1, 63, 64, 65, 2500, 4096, n - 2, n - 1]
    ck = starts(lk)
    pick = lambda t, c: torch.cat([t[c[i]:c[i + 1]] for i in some])
    plain = (pick(q, list(range(n + 1))), pick(k, ck), pick(v, ck), [1] * len(some), [lk[i] for i in some])
    got = ps.prompt_attention(q.cuda(), k.cuda(), v.cuda(), ints(range(n + 1)), ints(ck), max_q=1, max_k=max(lk))
    check(got.cpu()[some], *plain)
    store = ps.KV8(2 * n * page, Hk, D)
    place = torch.tensor([2 * page * i + j for i in range(n) for j in range(lk[i])], device="cuda")
    store.write(k.cuda(), v.cuda(), place)
    hk, hv = store.read(place, ps.F32)
    near = ps.prompt_attention(q.float().cuda(), hk, hv, ints(range(n + 1)), ints(ck), max_q=1)
    got = store.attention(q.float().cuda(), ints(range(n + 1)), ints(lk), ints([[2 * i, 2 * i + 1] for i in range(n)]), page, max_q=1, max_k=max(lk))
    # scores, softmax and sums of at most 30 keys in fp32, in two orders: 30 + 64 roundings of values below 6 each way
    assert torch.all((got - near).abs() <= 2 * 94 * 6 * 2.0 ** -24 * 8)
