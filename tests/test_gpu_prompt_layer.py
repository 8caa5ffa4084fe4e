"""The operators together: a layer of a causal text transformer over packed prompts, then one more token for each prompt."""
import pytest
import torch

import paper_2501_09253_amd as ps
import prompt_oracle as po
from test_gpu_prompt_attention import DT, ints, make, starts
from test_gpu_kv8 import CODE, paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_layer_then_single_tokens(dtype):
    C, H, Hk, D, page = 256, 4, 2, 64, 16
    lens = [77, 20, 130]
    n, T = len(lens), sum(lens)
    dt = DT[dtype]
    wqkv, wo, bo = make(1, (C, (H + 2 * Hk) * D), dt, C ** -0.5), make(2, (H * D, C), dt, C ** -0.5), make(3, (C,), dt)
    qkv_layer, out_layer = ps.Linear8(wqkv.cuda(), None, CODE[dtype]), ps.Linear8(wo.cuda(), bo.cuda(), CODE[dtype])
    table, places, total = paged([x + 1 for x in lens], page, 7)        # room for one more token each
    at = starts([x + 1 for x in lens])
    old = torch.cat([torch.arange(at[s], at[s] + lens[s]) for s in range(n)]).cuda()
    new = torch.tensor([at[s] + lens[s] for s in range(n)]).cuda()
    store = ps.KV8(total, Hk, D)

    def layer(x, cu, where, key_len, cached):
        qkv = qkv_layer.forward(x).view(x.shape[0], H + 2 * Hk, D)
        q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        store.write(k, v, places[where])
        o = store.attention(q, cu, key_len, table, page) if cached else ps.prompt_attention(q, k, v, cu)
        y = out_layer.forward(o.view(-1, H * D), res=x)
        return [t.clone() for t in (q, k, v, o, y)]

    x0, x1 = make(4, (T, C), dt).cuda(), make(5, (n, C), dt).cuda()
    q, k, v, o, y = layer(x0, ints(starts(lens)), old, None, False)
    q1, k1, v1, o1, y1 = layer(x1, ints(range(n + 1)), new, ints([x + 1 for x in lens]), True)

    def near(got, want, tol):
        assert torch.all((got.double().cpu() - want).abs() <= tol)

    def linear(x, w, b, res):
        (qx, sx), (qw, sw) = po.steps(x.cpu()), po.steps(w.t().contiguous())
        want = (qx @ qw.t()) * (sx * sw.t())
        size = want.abs()
        for t in (b, res):
            if t is not None:
                want, size = want + t.double().cpu(), size + t.double().cpu().abs()
        return want, 7 * po.U * size + po.HALF[dt] * want.abs()

    # every operator on what the one before it gave
    near(torch.cat([t.reshape(T, -1) for t in (q, k, v)], 1), *linear(x0, wqkv, None, None))
    near(y, *linear(o.reshape(T, -1), wo, bo, x0))
    near(y1, *linear(o1.reshape(n, -1), wo, bo, x1))
    cu = starts(lens)
    for s in range(n):
        r = slice(cu[s], cu[s + 1])
        out, bound, size = po.attention(q[r], k[r], v[r], D ** -0.5)
        near(o[r], out, po.attention_tolerance(out, bound, size, dt, D, lens[s]))
        kk, vv = (po.held(torch.cat([a[r], b[s:s + 1]]).cpu()) for a, b in ((k, k1), (v, v1)))
        out, bound, size = po.attention(q1[s:s + 1], kk, vv, D ** -0.5)
        near(o1[s:s + 1], out, po.attention_tolerance(out, bound, size, dt, D, lens[s] + 1) + 4 * po.U * bound)
