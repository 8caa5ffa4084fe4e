"""The 8-bit key/value store: what it holds, and the attention that reads it, against the plain 64-bit forms."""
import pytest
import torch

import paper_2501_09253_amd as ps
import prompt_oracle as po
from test_gpu_prompt_attention import DT, ints, make, starts

pytestmark = pytest.mark.gpu
CODE = {"bf16": ps.BF16, "f32": ps.F32}


def longs(values):
    return torch.tensor(values, dtype=torch.int64, device="cuda")


def same(got, want, dtype):
    """Whole number times scale: the scale and the product are rounded to fp32, the result to its type."""
    got, want = got.double().cpu(), want.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    err = (got - want).abs()
    tol = (2.5 * po.U + (po.HALF[dtype] if dtype == torch.bfloat16 else 0.0)) * want.abs()
    assert torch.all((err <= tol) | torch.isnan(want)), (err / tol).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,dim", [(8, 128), (2, 64), (1, 16), (3, 80), (5, 112)])
@pytest.mark.parametrize("rows", [1, 7, 128, 129, 1000])
def test_write_and_read(rows, heads, dim, dtype):
    k, v = make(1, (rows, heads, dim), DT[dtype]), make(2, (rows, heads, dim), DT[dtype], 30.0)
    store = ps.KV8(rows + 50, heads, dim)
    places = torch.randperm(rows + 50, generator=torch.Generator().manual_seed(3))[:rows].cuda()
    store.write(k.cuda(), v.cuda(), places)
    for out in ("bf16", "f32"):
        rk, rv = store.read(places, CODE[out])
        same(rk, po.held(k), DT[out])
        same(rv, po.held(v), DT[out])
    free = longs(sorted(set(range(rows + 50)) - set(places.tolist())))
    for t in store.read(free, ps.F32):
        assert torch.all(t == 0)


def test_borders_and_extremes():
    """Quotients on and next to the border of two numbers, tiny and huge values, zeros, infinities, NaN."""
    D = 64
    rows = []
    halves = torch.tensor([(2 * i + 1) / 254 for i in range(-32, 32)], dtype=torch.float64)
    for peak in (1.0, 127.0, 254.0, 3.5e37, 1.17e-37, 1e-44, 7.0 / 3):
        r = (halves * peak).float()
        r[0] = peak
        rows += [r, torch.nextafter(r, torch.full_like(r, float("inf"))), torch.nextafter(r, torch.full_like(r, float("-inf")))]
        rows[-1][0] = rows[-2][0] = peak
    rows += [torch.zeros(D), -torch.zeros(D), torch.full((D,), torch.finfo(torch.float32).max)]
    for bad in (float("inf"), float("-inf"), float("nan")):
        r = torch.linspace(-1, 1, D)
        r[9] = bad
        rows.append(r)
    k = torch.stack(rows).unsqueeze(1)
    store = ps.KV8(len(rows), 1, D)
    for x in (k, k.bfloat16()):
        store.write(x.cuda(), x.flip(0).contiguous().cuda(), torch.arange(len(rows), device="cuda"))
        got, back = store.read(torch.arange(len(rows), device="cuda"), ps.F32)
        q, s = po.steps(x)
        s = s.float().double()                                          # the scale is held in fp32, subnormal ones in few bits
        # 127 times the scale of the largest number, rounded up, lies above that number: the scale held is then one step (2 U of it)
        # smaller, and the value one more rounding away
        top = torch.finfo(torch.float32).max
        want, room = (q * s).clamp(-top, top), torch.where((q * s).abs() > top, 3.0, 1.0)
        ok = torch.isnan(want) | ((got.double().cpu() - want).abs() <= room * po.U * want.abs() + 2.0 ** -149)
        assert torch.all(ok) and torch.equal(torch.isnan(got.cpu()), torch.isnan(want))
        assert torch.equal(back.flip(0).isnan(), got.isnan()) and torch.equal(back.flip(0).nan_to_num(), got.nan_to_num())


@pytest.mark.parametrize("rows", [40, 700])
def test_places_left_out_and_taken_twice(rows):
    heads, D = 3, 64
    k, v = make(1, (rows, heads, D), torch.bfloat16), make(2, (rows, heads, D), torch.bfloat16)
    g = torch.Generator().manual_seed(5)
    places = torch.randint(0, rows // 3, (rows,), generator=g)
    places[3], places[rows - 1], places[5], places[7] = -1, rows + 10, 2 ** 40, -2 ** 60
    store = ps.KV8(rows + 10, heads, D)
    for _ in range(2):                                                  # nothing of the first call is left for the second
        store.write(k.cuda(), v.cuda(), places.cuda())
        last = {p: i for i, p in enumerate(places.tolist()) if 0 <= p < rows + 10}
        at = sorted(last)
        gk, gv = store.read(longs(at + [-1, rows + 10, 2 ** 50]), ps.F32)
        same(gk[:len(at)], po.held(k[[last[p] for p in at]]), torch.float32)
        same(gv[:len(at)], po.held(v[[last[p] for p in at]]), torch.float32)
        assert torch.all(gk[len(at):] == 0) and torch.all(gv[len(at):] == 0)
        k, v, places = v, k, places.flip(0)


def test_strided_rows():
    qkv = make(1, (30, 12, 64), torch.bfloat16).cuda()
    store, places = ps.KV8(40, 4, 64), torch.arange(3, 33, device="cuda")
    store.write(qkv[:, 4:8], qkv[:, 8:], places)
    gk, gv = store.read(places, ps.BF16)
    same(gk, po.held(qkv[:, 4:8].cpu()), torch.bfloat16)
    same(gv, po.held(qkv[:, 8:].cpu()), torch.bfloat16)


def paged(lk, page, seed, spare=3):
    """A table of shuffled pages and the place of every key, in packed order."""
    used = [-(-n // page) for n in lk]
    order = torch.randperm(sum(used) + spare, generator=torch.Generator().manual_seed(seed)).tolist()
    width = max(1, max(used))
    table, places = [], []
    for n, u in zip(lk, used):
        mine, order = order[:u], order[u:]
        table.append(mine + [-7] * (width - u))
        places += [mine[j // page] * page + j % page for j in range(n)]
    return ints(table), longs(places), (sum(used) + spare) * page


def check_cached(got, q, k, v, lq, lk, causal=True):
    D, dtype = q.shape[2], q.dtype
    got, cq, ck = got.double().cpu(), starts(lq), starts(lk)
    for s in range(len(lq)):
        out, bound, size = po.attention(q[cq[s]:cq[s + 1]], po.held(k[ck[s]:ck[s + 1]]), po.held(v[ck[s]:ck[s + 1]]), D ** -0.5, causal)
        tol = po.attention_tolerance(out, bound, size, dtype, D, lk[s]) + 4 * po.U * bound      # the values' scales
        err = (got[cq[s]:cq[s + 1]] - out).abs()
        assert torch.all(err <= tol), (s, lq[s], lk[s], (err / tol).max().item())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 64), (8, 2, 128), (3, 1, 80), (2, 1, 16), (6, 2, 32), (24, 1, 128)])
@pytest.mark.parametrize("page,lq,lk", [(16, [1, 1, 1, 1], [1, 16, 17, 300]), (1, [3, 1], [40, 5]), (64, [1, 20, 0, 2], [1500, 20, 9, 0]),
                                        (32, [5, 70], [3, 333]), (256, [130, 1], [130, 700])])
def test_attention_over_the_store(page, lq, lk, heads, kv_heads, dim, dtype):
    q, k, v = make(1, (sum(lq), heads, dim), DT[dtype]), make(2, (sum(lk), kv_heads, dim), DT[dtype]), make(3, (sum(lk), kv_heads, dim), DT[dtype])
    table, places, total = paged(lk, page, 4)
    store = ps.KV8(total, kv_heads, dim)
    store.write(k.cuda(), v.cuda(), places)
    for causal in (True, False):
        for hint in (0, max(lk)):
            got = store.attention(q.cuda(), ints(starts(lq)), ints(lk), table, page, causal=causal, max_q=max(lq), max_k=hint)
            check_cached(got, q, k, v, lq, lk, causal)


def test_what_the_store_holds_elsewhere_does_not_matter():
    """NaN groups behind the end, in pages of others; a NaN group inside reaches the queries that see it, no other."""
    lq, lk, H, Hk, D, page = [40, 1], [75, 200], 4, 2, 64, 16
    q, k, v = make(1, (sum(lq), H, D), torch.bfloat16), make(2, (sum(lk), Hk, D), torch.bfloat16), make(3, (sum(lk), Hk, D), torch.bfloat16)
    table, places, total = paged(lk, page, 4)
    store = ps.KV8(total, Hk, D)
    nan = torch.full((total, Hk, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    store.write(nan, nan, torch.arange(total, device="cuda"))
    store.write(k.cuda(), v.cuda(), places)
    run = lambda: store.attention(q.cuda(), ints(starts(lq)), ints(lk), table, page)
    want = run()
    check_cached(want, q, k, v, lq, lk)
    for side in (0, 1):
        kv = [k[60:61].cuda(), v[60:61].cuda()]
        kv[side] = nan[:1]
        store.write(*kv, places[60:61])                                 # key 60: queries 25 .. of the first sequence see it
        got = run()
        assert torch.equal(got[:25], want[:25]) and torch.equal(got[40:], want[40:]) and torch.isnan(got[25:40]).all()
        store.write(k[60:61].cuda(), v[60:61].cuda(), places[60:61])
        assert torch.equal(run(), want)


def test_pages_outside_and_lengths_past_the_table():
    """Keys on pages that are none of the store's count as not there; a length past the table is cut to it."""
    H, Hk, D, page = 2, 1, 64, 16
    k, v, q = make(2, (64, Hk, D), torch.bfloat16), make(3, (64, Hk, D), torch.bfloat16), make(1, (2, H, D), torch.bfloat16)
    store = ps.KV8(64, Hk, D)
    store.write(k.cuda(), v.cuda(), torch.arange(64, device="cuda"))
    got = store.attention(q.cuda(), ints([0, 1, 2]), ints([50, 1000]), ints([[2, -1, 1, 99], [0, 1, 2, 2 ** 30]]), page)
    here = [list(range(32, 48)) + list(range(16, 32)), list(range(48))]
    for s in range(2):
        out, bound, size = po.attention(q[s:s + 1], po.held(k[here[s]]), po.held(v[here[s]]), D ** -0.5, False)
        tol = po.attention_tolerance(out, bound, size, q.dtype, D, 64) + 4 * po.U * bound
        assert torch.all((got[s:s + 1].double().cpu() - out).abs() <= tol)
    none = store.attention(q.cuda(), ints([0, 1, 2]), ints([0, 40]), ints([[0], [-3]]), page)
    assert torch.all(none == 0)


def test_a_long_sequence_of_single_tokens():
    """Token by token: write the new token, attend, against the whole prompt at once; captured into a graph for some of the steps."""
    H, Hk, D, page, n = 8, 2, 128, 32, 3
    L = 70
    q, k, v = make(1, (n, L, H, D), torch.bfloat16).cuda(), make(2, (n, L, Hk, D), torch.bfloat16).cuda(), make(3, (n, L, Hk, D), torch.bfloat16).cuda()
    pages = -(-L // page)
    table = torch.randperm(n * pages, generator=torch.Generator().manual_seed(1)).view(n, pages).int().cuda()
    place = lambda t: table[:, t // page].long() * page + t % page
    store, cu = ps.KV8(n * pages * page, Hk, D), ints([0, 1, 2, 3])
    qs, ks, vs, at, lens = q[:, 0].clone(), k[:, 0].clone(), v[:, 0].clone(), place(0).clone(), ints([1] * n)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(qs)

    def step():
        store.write(ks, vs, at)
        store.attention(qs, cu, lens, table, page, max_q=1, max_k=L, out=out, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    steps = []
    for t in range(L):
        for dst, src in ((qs, q[:, t]), (ks, k[:, t]), (vs, v[:, t]), (at, place(t))):
            dst.copy_(src)
        lens.fill_(t + 1)
        graph.replay() if t % 3 else step()
        steps.append(out.clone())
    got = torch.stack(steps, 1).reshape(n * L, H, D)
    check_cached(got, q.reshape(n * L, H, D).cpu(), k.reshape(n * L, Hk, D).cpu(), v.reshape(n * L, Hk, D).cpu(), [L] * n, [L] * n)
