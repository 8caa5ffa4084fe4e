"""The operators together, as a transformer layer over a mixed-resolution batch with text uses them: norm into 8 bits, q/k/v in 8-bit floating point,
positions, attention over each request's tokens, output layer, gate and residual with the next sub-layer's norm."""
import pytest
import torch

import layer_oracle as lo
import paper_2501_09253_amd as ps
import prompt_oracle as po
from test_gpu_gated_norm import near, near8
from test_gpu_kv8 import CODE
from test_gpu_prompt_attention import DT, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("graph", [False, True])
def test_a_layer_over_a_joint_plan(dtype, graph):
    C, H, D, dt = 256, 4, 64, DT[dtype]
    plan = ps.Plan([(8, 8), (8, 16), (16, 8)], 4, 4, text_len=20)
    T, n = plan.T, plan.n
    wqkv, wo, bo = make(1, (C, 3 * H * D), dt, C ** -0.5), make(2, (H * D, C), dt, C ** -0.5), make(3, (C,), dt)
    qkv_layer, out_layer = ps.LinearF8(wqkv.cuda(), None, CODE[dtype]), ps.LinearF8(wo.cuda(), bo.cuda(), CODE[dtype])
    mod = make(4, (n, 3 * C), dt, 0.3).cuda()
    gate, scale, shift = mod.chunk(3, dim=1)
    g1, g2, g3 = ((1 + make(5 + i, (C,), torch.float32, 0.2)).to(dt).cuda() for i in range(3))
    axis, freq = ps.rotary_ladder((8, 12, 12))
    rot = ps.Rotary(axis, freq, "next")
    pos = plan.positions(torch.arange(n, dtype=torch.float32, device="cuda"), [0, 0, 0, 1, 1, 1])
    cu = torch.from_numpy(plan.table("cu_seqlens").copy()).cuda()
    x = make(9, (T, C), dt).cuda()
    rows8, ws = ps.RowsF8(T, C), torch.empty(out_layer.workspace_bytes(T), dtype=torch.uint8, device="cuda")
    h, y, o = (torch.empty((T, C), dtype=dt, device="cuda") for _ in range(3))
    qkv, out = torch.empty((T, 3 * H * D), dtype=dt, device="cuda"), torch.empty((T, C), dtype=dt, device="cuda")
    turned = torch.empty((T, 2 * H, D), dtype=dt, device="cuda")

    def layer():
        ps.gated_norm(x, pre="layer", pre_gain=g1, scale=scale, shift=shift, plan=plan, rows8=rows8)
        qkv_layer.forward(rows8, y=qkv)
        q, k, v = qkv.view(T, 3, H, D).unbind(1)
        rot.forward(q, k, pos, q_out=turned[:, :H], k_out=turned[:, H:])
        ps.prompt_attention(turned[:, :H], turned[:, H:], v, cu, causal=False, out=o.view(T, H, D))
        out_layer.forward(o, y=out, workspace=ws)
        ps.gated_norm(x, out, post="rms", post_gain=g2, gate=gate, pre="rms", pre_gain=g3, plan=plan, y=y, h=h)

    layer()
    if graph:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            layer()
        for seed in (20, 21, 22):
            x.copy_(make(seed, (T, C), dt))
            layer()
            eager = [t.clone() for t in (qkv, turned, o, out, y, h)]
            for t in (qkv, turned, o, out, y, h):
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(eager, (qkv, turned, o, out, y, h)):
                assert torch.equal(a, b)

    # every operator on what the one before it gave
    request = torch.cat([torch.full((int(cu[s + 1] - cu[s]),), int(plan.table("perm")[s])) for s in range(n)])
    _, want = lo.gated_norm(x, pre="layer", pre_gain=g1, scale=scale, shift=shift, request=request)
    near8(rows8, want)
    held = rows8.read(CODE[dtype]).cpu()
    want, tol, _ = lo.linear_f8(held, wqkv, None, None, dt)
    assert torch.all((qkv.double().cpu() - want).abs() <= tol)
    q, k, v = qkv.view(T, 3, H, D).unbind(1)
    for got, src in ((turned[:, :H], q), (turned[:, H:], k)):
        want, bound = lo.rotary(src, pos, axis, freq, False)
        assert torch.all((got.double().cpu() - want).abs() <= bound + lo.HALF[dt] * want.abs())
    for s in range(n):
        r = slice(int(cu[s]), int(cu[s + 1]))
        want, bound, size = po.attention(turned[r, :H], turned[r, H:], v[r], D ** -0.5, causal=False)
        tol = po.attention_tolerance(want, bound, size, dt, D, r.stop - r.start)
        assert torch.all((o.view(T, H, D)[r].double().cpu() - want).abs() <= tol)
    want, tol, _ = lo.linear_f8(o.cpu(), wo, bo, None, dt)
    assert torch.all((out.double().cpu() - want).abs() <= tol)
    wy, wh = lo.gated_norm(x, out, post="rms", post_gain=g2, gate=gate, pre="rms", pre_gain=g3, request=request)
    near(y, wy, dtype)
    near(h, wh, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C,N", [(40, 640, 200), (40, 4100, 130), (300, 2048, 640), (700, 640, 768), (5000, 384, 3400), (8000, 600, 4001)])
def test_rows_that_were_never_written(rows, C, N, dtype):
    """What rows of no request hold in new 8-bit rows, numbers and powers of two that are NaN among it, has no part in the other rows' results."""
    dt = DT[dtype]
    x, layer = make(1, (rows, C), dt).cuda(), ps.LinearF8(make(2, (C, N), dt, C ** -0.5).cuda(), None, CODE[dtype])
    cu = torch.tensor([1, rows // 2, rows - 2], dtype=torch.int32, device="cuda")
    want = None
    for fill in (0, 255, 127, 254):
        rows8 = ps.RowsF8(rows, C)
        rows8.buffer.fill_(fill)
        ps.gated_norm(x, pre="rms", cu_rows=cu, rows8=rows8)
        got = layer.forward(rows8)[1:rows - 2]
        want = got if want is None else want
        assert torch.isfinite(got).all() and torch.equal(got, want)
