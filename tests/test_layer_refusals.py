"""CPU-only: what the layer-side entry points refuse (no kernel is launched, no pointer is read)."""
import ctypes as C

import pytest
import torch

import layer_oracle as lo
import paper_2501_09253_amd as ps
from paper_2501_09253_amd import binding
from test_prompt_refusals import P, refused


def test_rotary_create_refuses():
    L, out = ps.lib(), C.c_void_p()
    axis, freq = (C.c_int32 * 4)(0, 1, 1, 2), (C.c_double * 4)(1, 1, 1, 1)
    refused(L.pserve_rotary_create(3, 4, axis, freq, 0, None, None), "NULL")
    refused(L.pserve_rotary_create(3, 4, None, freq, 0, None, C.byref(out)), "NULL")
    refused(L.pserve_rotary_create(3, 4, axis, None, 0, None, C.byref(out)), "NULL")
    for axes, pairs, layout, word in ((0, 4, 0, "axes"), (9, 4, 0, "axes"), (3, 0, 0, "pairs"), (3, 257, 0, "pairs"), (3, 4, 2, "layout"), (2, 4, 0, "axis 2")):
        refused(L.pserve_rotary_create(axes, pairs, axis, freq, layout, None, C.byref(out)), word)
    for bad in (float("nan"), float("inf"), 2e9):
        refused(L.pserve_rotary_create(3, 4, axis, (C.c_double * 4)(1, 1, bad, 1), 0, None, C.byref(out)), "pair 2")
    assert not out.value
    for axis, freq, kw, word in (([], [], {}, "each pair"), ([0], [1.0, 2.0], {}, "each pair"), ([0], [1.0], dict(layout="both"), "layout"), ([-1], [1.0], dict(axes=2), "axis")):
        with pytest.raises(ps.PserveError, match=word):
            ps.Rotary(axis, freq, **kw)


def rotary_desc(**change):
    d = binding._RotaryDesc(4, 2, 64, ps.BF16, 10)
    d.q_stride[:], d.k_stride[:], d.q_out_stride[:], d.k_out_stride[:] = (256, 64), (128, 64), (256, 64), (128, 64)
    for k, v in change.items():
        if isinstance(v, tuple):
            getattr(d, k)[:] = v
        else:
            setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,word", [
    (dict(heads=0), "heads"), (dict(heads=4097), "heads"), (dict(kv_heads=-1), "heads"), (dict(head_dim=62), "head_dim"), (dict(head_dim=513), "head_dim"),
    (dict(dtype=2), "dtype"), (dict(tokens=-1), "tokens"), (dict(tokens=2 ** 31), "tokens"), (dict(q_stride=(-1, 64)), "stride"),
    (dict(k_stride=(128, 2 ** 31)), "stride"), (dict(q_out_stride=(2 ** 40, 64)), "stride"), (dict(k_out_stride=(128, -64)), "stride")])
def test_rotary_refuses(change, word):
    L = ps.lib()
    op = (C.c_int64 * 64)()
    op[0], op[1] = 3 | 32 << 32, 0                              # axes, pairs; layout (an image of the fields the checks read)
    refused(L.pserve_rotary_forward(op, C.byref(rotary_desc(**change)), P, P, P, P, P, None), word)


def test_rotary_buffers():
    L, d = ps.lib(), rotary_desc()
    op = (C.c_int64 * 64)()
    op[0] = 3 | 32 << 32
    refused(L.pserve_rotary_forward(None, C.byref(d), P, P, P, P, P, None), "NULL")
    refused(L.pserve_rotary_forward(op, None, P, P, P, P, P, None), "NULL")
    for i in range(5):
        args = [P] * 5
        args[i] = None
        refused(L.pserve_rotary_forward(op, C.byref(d), *args, None), "NULL")
        args[i] = P + 1
        refused(L.pserve_rotary_forward(op, C.byref(d), *args, None), "aligned")
    assert L.pserve_rotary_forward(op, C.byref(rotary_desc(tokens=0)), None, None, None, None, None, None) == 0
    refused(L.pserve_plan_positions(None, None, None, P, None), "NULL")


def norm_call(desc=None, **buffers):
    d = binding._GatedNormDesc(64, ps.BF16, 1, 1, 2, 1e-5, 1e-5, 1.0, 1.0, 10, *[64] * 7)
    for k, v in (desc or {}).items():
        setattr(d, k, v)
    b = binding._GatedNormBuffers(x=P, f=P, y=P, h=P)
    for k, v in buffers.items():
        setattr(b, k, v)
    return ps.lib().pserve_gated_norm(C.byref(d), C.byref(b), None)


@pytest.mark.parametrize("desc,buffers,word", [
    (dict(C=0), {}, "channels"), (dict(C=16385), {}, "channels"), (dict(dtype=3), {}, "dtype"), (dict(n=0), {}, "n > 0"), (dict(n=2), {}, "cu_rows"),
    (dict(post_norm=3), {}, "norm"), (dict(pre_norm=-1), {}, "norm"), (dict(post_eps=-1.0), {}, "eps"), (dict(pre_eps=float("nan")), {}, "eps"),
    (dict(branch_scale=float("inf")), {}, "scale"), (dict(skip_scale=float("nan")), {}, "scale"), (dict(rows=-1), {}, "rows"), (dict(rows=2 ** 31), {}, "rows"),
    (dict(x_stride=63), {}, "stride"), (dict(f_stride=-64), {}, "stride"), (dict(h_stride=2 ** 31), {}, "stride"), (dict(gate_stride=-1), dict(gate=P), "stride"),
    ({}, dict(x=None), "NULL"), (dict(pre_norm=0), dict(y=None, h=None), "NULL"), ({}, dict(f=None), "without its output"), ({}, dict(h=None), "without h"),
    ({}, dict(rows8=P), "at once"), ({}, dict(h=None, rows8=P + 4), "aligned"), ({}, dict(x=P + 1), "aligned"), ({}, dict(shift=P + 1), "aligned"),
    (dict(post_norm=0), dict(f=None, gate=P), "without its output"), (dict(pre_norm=0), dict(h=None, scale=P), "without h")])
def test_gated_norm_refuses(desc, buffers, word):
    refused(norm_call(desc, **buffers), word)


def test_gated_norm_arguments():
    refused(ps.lib().pserve_gated_norm(None, None, None), "NULL")
    assert norm_call(dict(rows=0), x=None, f=P, y=None) == 0


def test_rows_and_layers_refuse():
    L, out, need = ps.lib(), C.c_void_p(), C.c_size_t()
    for rows, K in ((-1, 8), (1 << 26, 8), (8, 0), (8, 131073)):
        refused(L.pserve_f8_rows_bytes(rows, K, C.byref(need)), "rows" if K == 8 else "K =")
    refused(L.pserve_f8_rows_bytes(4, 8, None), "NULL")
    assert L.pserve_f8_rows_bytes(3, 600, C.byref(need)) == 0 and need.value == 3 * (640 + 8)
    for call in (lambda x, r8, rows=4, ldx=8, dt=1: L.pserve_f8_rows_write(x, ldx, rows, 8, dt, r8, None),
                 lambda x, r8, rows=4, ldx=8, dt=1: L.pserve_f8_rows_read(r8, rows, 8, dt, x, ldx, None)):
        refused(call(None, P), "NULL")
        refused(call(P, None), "NULL")
        refused(call(P, P + 8), "aligned")
        refused(call(P + 1, P), "aligned")
        refused(call(P, P, ldx=7), "apart")
        refused(call(P, P, dt=2), "dtype")
        refused(call(P, P, rows=-1), "rows")
        assert call(None, None, rows=0) == 0
    for K, N, dtype, w in ((0, 8, 1, P), (8, 0, 1, P), (131073, 8, 1, P), (8, (1 << 24) + 1, 1, P), (8, 8, 5, P), (8, 8, 1, None), (8, 8, 1, P + 1)):
        assert L.pserve_linear_f8_create(K, N, dtype, w, None, None, C.byref(out)) == -1 and not out.value
    refused(L.pserve_linear_f8_create(8, 8, 1, P, None, None, None), "NULL")
    refused(L.pserve_linear_f8_forward(None, P, 8, 4, None, P, 1000, P, None), "NULL")
    refused(L.pserve_linear_f8_forward_rows(None, P, 4, None, P, None), "NULL")
    refused(L.pserve_linear_f8_workspace(None, 4, C.byref(need)), "NULL")
    layer = (C.c_int64 * 64)()                                  # an image of the fields that the checks read: K, N; rounded up; dtype
    layer[0], layer[1], layer[2] = 100 | 8 << 32, 128 | 256 << 32, 1
    assert L.pserve_linear_f8_workspace(layer, 40000, C.byref(need)) == 0 and need.value == 40000 * 132
    assert L.pserve_linear_f8_workspace(layer, 5, C.byref(need)) == 0 and need.value == 0      # (rounded on the way in)
    refused(L.pserve_linear_f8_workspace(layer, 1 << 26, C.byref(need)), "rows")
    refused(L.pserve_linear_f8_forward(layer, P, 99, 40000, None, P, 5280000, P, None), "apart")
    refused(L.pserve_linear_f8_forward(layer, P, 100, 40000, None, P, 5279999, P, None), "workspace")
    refused(L.pserve_linear_f8_forward(layer, P, 100, 40000, None, P + 8, 5280000, P, None), "workspace")
    refused(L.pserve_linear_f8_forward(layer, P, 100, 40000, None, None, 5280000, P, None), "NULL")
    refused(L.pserve_linear_f8_forward_rows(layer, P + 4, 5, None, P, None), "aligned")
    refused(L.pserve_linear_f8_forward_rows(layer, None, 5, None, P, None), "NULL")
    assert L.pserve_linear_f8_forward(layer, None, 100, 0, None, None, 0, None, None) == 0


def test_binding_refuses_tensors_that_are_not_on_the_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ps.PserveError, match="device"):
        ps.gated_norm(torch.zeros(4, 8), pre="rms")
    with pytest.raises(ps.PserveError, match="device"):
        ps.LinearF8(torch.zeros(8, 8), None, ps.F32)


@pytest.fixture
def anywhere(monkeypatch):
    monkeypatch.setattr(binding, "_here", lambda *a: None)


def test_gated_norm_binding(anywhere):
    x, v = torch.zeros(4, 8), torch.zeros(8)
    for kw, word in ((dict(post="batch"), "norm"), (dict(pre_gain=torch.zeros(7), pre="rms"), "gains"), (dict(gate=torch.zeros(2, 8), f=x), "gate"),
                     (dict(f=torch.zeros(4, 9)), "must be"), (dict(f=x.bfloat16()), "must be"), (dict(cu_rows=torch.zeros(3)), "cu_rows"),
                     (dict(cu_rows=torch.zeros(1, dtype=torch.int32)), "cu_rows"), (dict(which=torch.zeros(2, dtype=torch.int32)), "which"),
                     (dict(pre="rms", h=x[:, :].t()), "must be"), (dict(f=x.expand(4, 8)[:1].expand(4, 8)), "must be")):
        with pytest.raises(ps.PserveError, match=word):
            ps.gated_norm(x, **kw)
    buf = torch.zeros(9, 8)
    for kw in (dict(y=buf[1:5]), dict(f=buf[4:8], y=buf[5:9]), dict(y=buf[4:8], h=buf[4:8], pre="rms"), dict(h=buf[2:6], pre="rms")):
        with pytest.raises(ps.PserveError, match="overlap"):
            ps.gated_norm(buf[:4], **kw)
    with pytest.raises(ps.PserveError, match="overlap"):
        ps.gated_norm(x[:1], pre="rms", pre_gain=v, h=v.view(1, 8))


def test_rotary_binding(anywhere):
    rot = ps.Rotary.__new__(ps.Rotary)
    rot._h, rot.pairs, rot.axes = C.c_void_p(), 4, 2
    q, k, pos = torch.zeros(6, 4, 8), torch.zeros(6, 2, 8), torch.zeros(6, 2)
    for args, kw, word in (((q, k, torch.zeros(6, 3)), {}, "pos"), ((q, k, pos.double()), {}, "pos"), ((q, k[:5], pos), {}, "one dtype"), ((q, k.bfloat16(), pos), {}, "one dtype"),
                           ((q[0], k, pos), {}, "one dtype"), ((q.half(), None, pos), {}, "dtype"), ((q, None, pos), dict(k_out=k), "without k"),
                           ((q.transpose(1, 2), None, pos), {}, "consecutive"), ((q, None, pos), dict(q_out=q[:, :2]), "shape"),
                           ((q, None, pos), dict(q_out=torch.zeros(6, 1, 8).expand(6, 4, 8)), "overlap")):
        with pytest.raises(ps.PserveError, match=word):
            rot.forward(*args, **kw)
    buf = torch.zeros(13, 4, 8)
    for qo, ko in ((buf[1:7], None), (None, buf[:6, :2]), (buf[6:12], buf[7:13, :2])):
        with pytest.raises(ps.PserveError, match="overlap"):
            rot.forward(buf[:6], k, pos, q_out=qo, k_out=ko)


def test_heads_side_by_side():
    m = torch.zeros(5, 9, 8)
    q, k, v = m[:, :4], m[:, 4:6], m[:, 6:]
    assert binding._interleaved(q, k) and binding._interleaved(k, q) and binding._interleaved(v, q)
    assert not binding._interleaved(q, m[:, 3:5]) and not binding._interleaved(m[:, 3:5], q) and not binding._interleaved(q, q)
    flat = torch.zeros(400)
    a = flat[:5 * 72].view(5, 9, 8)[:, :4]
    assert not binding._interleaved(a, flat[50:50 + 320].as_strided((4, 4, 8), (72, 8, 1), 50))      # runs over the row's end into a's next one
    assert binding._interleaved(a, flat.as_strided((4, 4, 8), (72, 8, 1), 32))


def test_the_oracle_rounds_as_torch_does():
    """The format's rounding in the oracle against torch's conversion."""
    x = torch.randn(20000, generator=torch.Generator().manual_seed(1)) * torch.exp2(torch.randint(-12, 8, (20000,), generator=torch.Generator().manual_seed(2)).float())
    x = torch.cat([x.clamp(-448, 448), torch.arange(0, 449 * 64) / 64.0, torch.arange(0, 64) * 2.0 ** -11])
    _, r = lo.f8_round(x.double())
    assert torch.equal(r.float(), x.to(torch.float8_e4m3fn).float())


def test_bounds_catch_a_block_left_out():
    """A block of 128 left out, counted twice or taken with half its scale breaks the layer's bounds, so does a norm over one value less."""
    for dtype in (torch.bfloat16, torch.float32):
        g = torch.Generator().manual_seed(3)
        x, w = torch.randn((64, 1024), generator=g).to(dtype), (torch.randn((1024, 80), generator=g) / 32).to(dtype)
        want, tol, _ = lo.linear_f8(x, w, None, None, dtype)
        hx, hw = lo.f8_held(x)[2], lo.f8_held(w.t().contiguous())[2]
        block = hx[:, 384:512] @ hw[:, 384:512].t()
        for wrong in (want - block, want + block, want - block / 2):
            assert not torch.all((wrong - want).abs() <= tol)
    x = torch.randn((8, 256), generator=g)
    _, h = lo.gated_norm(x, pre="rms")
    _, less = lo.gated_norm(x[:, :255], pre="rms")
    assert not torch.all((less.v - h.v[:, :255]).abs() <= h.e[:, :255] + lo.HALF[torch.float32] * h.v[:, :255].abs())
