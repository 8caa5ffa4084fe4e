"""Rotary positions with several axes against the plain 64-bit form, value by value within the bound of tests/layer_oracle.py."""
import math

import numpy as np
import pytest
import torch

import layer_oracle as lo
import paper_2501_09253_amd as ps
from test_gpu_prompt_attention import DT, make

pytestmark = pytest.mark.gpu


def positions(seed, tokens, axes, far=200.0):
    return (torch.rand((tokens, axes), generator=torch.Generator().manual_seed(seed)) * far).round()


def check(got, x, pos, axis, freq, half):
    want, bound = lo.rotary(x, pos, axis, freq, half)
    tol = bound + lo.HALF[x.dtype] * want.abs() + 1e-37
    err = (got.double().cpu() - want).abs()
    assert torch.all(err <= tol), (err / tol).max().item()


# heads, kv_heads, dim, pairs of each axis
HEADS = [(4, 4, 64, (8, 12, 12)), (8, 2, 128, (16, 24, 24)), (3, 1, 80, (8, 12, 12)), (2, 1, 16, (8,)), (6, 2, 32, (2, 3, 3)), (5, 5, 96, (12, 18, 18)),
         (1, 1, 2, (1,)), (2, 2, 10, (1, 2)), (3, 2, 17, (4, 3)), (2, 1, 256, (64, 32, 16, 16)), (1, 1, 512, (100, 156)), (40, 8, 64, (5, 27)), (4, 2, 24, (8,)),
         (130, 2, 64, (16, 16))]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "next"])
@pytest.mark.parametrize("heads,kv_heads,dim,pairs", HEADS)
def test_head_layouts(heads, kv_heads, dim, pairs, layout, dtype):
    axis, freq = ps.rotary_ladder(pairs, 10000.0, shared=len(pairs) == 2)
    rot = ps.Rotary(axis, freq, layout)
    for tokens in (1, 3, 37, 300):
        q, k, pos = make(1, (tokens, heads, dim), DT[dtype]), make(2, (tokens, kv_heads, dim), DT[dtype]), positions(3, tokens, len(pairs))
        gq, gk = rot.forward(q.cuda(), k.cuda(), pos.cuda())
        check(gq, q, pos, axis, freq, layout == "half")
        check(gk, k, pos, axis, freq, layout == "half")
        alone, none = rot.forward(q.cuda(), None, pos.cuda())
        assert none is None and torch.equal(alone, gq)


@pytest.mark.parametrize("tokens", [1, 2, 63, 64, 65, 1000, 20000])
def test_lengths(tokens):
    axis, freq = ps.rotary_ladder((8, 12, 12))
    rot = ps.Rotary(axis, freq)
    q, k, pos = make(1, (tokens, 3, 64), torch.bfloat16), make(2, (tokens, 1, 64), torch.bfloat16), positions(3, tokens, 3, 5000)
    gq, gk = rot.forward(q.cuda(), k.cuda(), pos.cuda())
    check(gq, q, pos, axis, freq, True)
    check(gk, k, pos, axis, freq, True)


@pytest.mark.parametrize("layout", ["half", "next"])
def test_offsets_past_32_bits(layout):
    """2.5e9 values in and out: the last tokens are what they are in a call of their own."""
    T, H, D = 300000, 64, 128
    axis, freq = ps.rotary_ladder((16, 24, 24))
    rot = ps.Rotary(axis, freq, layout)
    q = torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda")
    q.view(-1, 100, H, D)[:] = make(1, (100, H, D), torch.bfloat16).cuda()
    q[-3:] *= 2
    pos = positions(2, T, 3, 1e5).cuda()
    got, _ = rot.forward(q, None, pos)
    for part in (slice(T - 50, T), slice(T // 2, T // 2 + 50)):
        assert torch.equal(got[part], rot.forward(q[part].clone(), None, pos[part].contiguous())[0])


def test_no_tokens():
    rot = ps.Rotary([0], [1.0])
    q = torch.empty((0, 2, 8), dtype=torch.float32, device="cuda")
    gq, _ = rot.forward(q, None, torch.empty((0, 1), device="cuda"))
    assert gq.shape == q.shape


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "next"])
def test_far_fractional_and_negative_positions(layout, dtype):
    """Angles of 16 million radians: 32 bits would leave them off by one."""
    axis, freq = [0, 1, 1, 2, 0, 2, 1, 0], [1.0, 1.0, 0.731, 1e-4, 2.5, 1e3, 1e-9, math.pi]
    rot = ps.Rotary(axis, freq, layout, axes=4)                 # (an axis that no pair uses)
    pos = torch.cat([positions(1, 30, 4, 2.0 ** 24), -positions(2, 30, 4, 2.0 ** 20), torch.rand((40, 4), generator=torch.Generator().manual_seed(3)) * 100 - 50])
    q = make(4, (100, 2, 20), DT[dtype])
    gq, _ = rot.forward(q.cuda(), None, pos.cuda())
    check(gq, q, pos, axis, freq, layout == "half")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "next"])
@pytest.mark.parametrize("dim,off", [(64, 0), (64, 8), (64, 3), (40, 0)])
def test_strides_and_in_place(dim, off, layout, dtype):
    """Queries and keys inside one matrix of a projection, heads inside tokens and tokens inside heads, out of place and in place."""
    T, H, Hk = 70, 6, 2
    axis, freq = ps.rotary_ladder((4, 8, 6))
    rot = ps.Rotary(axis, freq, layout)
    pos = positions(5, T, 3)
    wide = make(6, (T, (H + 2 * Hk) * dim + off), DT[dtype])
    qkv = wide.cuda()[:, off:].view(T, H + 2 * Hk, dim)
    q, k = qkv[:, :H], qkv[:, H:H + Hk]
    hq, hk = q.cpu(), k.cpu()
    gq, gk = rot.forward(q, k, pos.cuda())
    check(gq, hq, pos, axis, freq, layout == "half")
    check(gk, hk, pos, axis, freq, layout == "half")
    v = qkv[:, H + Hk:].clone()
    rot.forward(q, k, pos.cuda(), q_out=q, k_out=k)
    assert torch.equal(q, gq) and torch.equal(k, gk) and torch.equal(qkv[:, H + Hk:], v)
    by_head = hq.permute(1, 0, 2).contiguous().cuda().permute(1, 0, 2)      # [H][T][D]
    out = torch.full((H, T + 2, dim + 16), 7.0, dtype=DT[dtype], device="cuda")
    view = out[:, 1:T + 1, 8:8 + dim].permute(1, 0, 2)
    rot.forward(by_head, None, pos.cuda(), q_out=view)
    assert torch.equal(view, gq)
    view.fill_(7)
    assert torch.all(out == 7)                                  # nothing beside it was written
    wide_out = torch.empty((T, H + Hk, dim), dtype=DT[dtype], device="cuda")     # two outputs side by side
    rot.forward(hq.cuda(), hk.cuda(), pos.cuda(), q_out=wide_out[:, :H], k_out=wide_out[:, H:])
    assert torch.equal(wide_out[:, :H], gq) and torch.equal(wide_out[:, H:], gk)


@pytest.mark.parametrize("layout", ["half", "next"])
def test_what_is_not_finite_stays_in_its_pairs(layout):
    axis, freq = [0, 1, 0, 1, 1, 0, 0, 1], [1.0, 1.0, 0.5, 0.5, 0.1, 0.1, 0.01, 0.01]
    rot = ps.Rotary(axis, freq, layout)
    q, pos = make(1, (5, 3, 24), torch.float32), positions(2, 5, 2)
    clean, _ = rot.forward(q.cuda(), None, pos.cuda())
    bad = pos.clone()
    bad[1, 0], bad[2, 1], bad[3, 0] = float("nan"), float("inf"), float("-inf")
    got, _ = rot.forward(q.cuda(), None, bad.cuda())
    for t in range(5):
        for p in range(8):
            pair = [p, p + 8] if layout == "half" else [2 * p, 2 * p + 1]
            if math.isfinite(bad[t, axis[p]]):
                assert torch.equal(got[t][:, pair], clean[t][:, pair])
            else:
                assert torch.isnan(got[t][:, pair]).all()
    assert torch.equal(got[:, :, 16:], q[:, :, 16:].cuda())     # behind the pairs: copied
    q2 = q.clone()
    q2[0, 1, 3], q2[4, 2, 20], q2[4, 0, 23] = float("inf"), float("nan"), float("-inf")
    got, _ = rot.forward(q2.cuda(), None, pos.cuda())
    p = 3 if layout == "half" else 1
    pair = [p, p + 8] if layout == "half" else [2 * p, 2 * p + 1]
    assert not torch.isfinite(got[0, 1, pair]).any()
    keep = torch.ones_like(q, dtype=torch.bool)
    keep[0, 1, pair] = False
    keep[:, :, 16:] = False
    assert torch.equal(got[keep.cuda()], clean[keep.cuda()])
    assert torch.equal(got[:, :, 16:].nan_to_num(9.0), q2[:, :, 16:].nan_to_num(9.0).cuda())


@pytest.mark.parametrize("res,ph,pw,text", [([(16, 16), (8, 24), (16, 8)], 8, 8, 0), ([(16, 16), (8, 24), (16, 8)], 8, 8, 77), ([(12, 6), (6, 6)], 3, 2, 7), ([(5, 7)], 5, 7, 1)])
def test_positions_of_a_plan(res, ph, pw, text):
    plan = ps.Plan(res, ph, pw, text_len=text)
    frame = torch.arange(len(res), dtype=torch.float32) + 10
    steps = [1.0, 2.0, 3.0, 0.5, 1.0, -1.0]
    got = plan.positions(frame.cuda(), steps).cpu().numpy()
    assert got.shape == (plan.T, 3)
    owner, rc, perm, S = plan.table("patch_owner"), plan.table("patch_rc"), plan.table("perm"), ph * pw
    want = np.zeros_like(got)
    for t in range(plan.T):
        p, r = divmod(t, S)
        row, col = rc[p]
        if row < 0:
            j = col * S + r
            if j < text:
                want[t] = [steps[i] + j * steps[3 + i] for i in range(3)]
        else:
            want[t] = [frame[perm[owner[p]]], row * ph + r // pw, col * pw + r % pw]
    assert np.array_equal(got, want)
    plain = plan.positions().cpu().numpy()
    want[:, 0] = 0
    for t in range(plan.T):
        if rc[t // S][0] < 0:
            want[t] = 0
    assert np.array_equal(plain, want)


def test_graph_and_streams():
    axis, freq = ps.rotary_ladder((8, 12, 12))
    rot = ps.Rotary(axis, freq)
    q, k, pos = make(1, (200, 4, 64), torch.bfloat16).cuda(), make(2, (200, 2, 64), torch.bfloat16).cuda(), positions(3, 200, 3).cuda()
    want = rot.forward(q, k, pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = rot.forward(q, k, pos)
    side.synchronize()
    assert torch.equal(other[0], want[0]) and torch.equal(other[1], want[1])
    oq, ok = torch.empty_like(q), torch.empty_like(k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rot.forward(q, k, pos, q_out=oq, k_out=ok)
    for i in range(3):
        q.copy_(make(20 + i, (200, 4, 64), torch.bfloat16))
        pos.copy_(positions(30 + i, 200, 3))
        graph.replay()
        torch.cuda.synchronize()
        want = rot.forward(q, k, pos)
        assert torch.equal(oq, want[0]) and torch.equal(ok, want[1])


def test_far_angles_within_what_the_header_says():
    """Angles around 2^35 radians against whole-number arithmetic: 3 * 2^-53 of an angle (three roundings in 64 bits; 2^-52 is passed), 2^-22 of a sine and cosine."""
    from fractions import Fraction
    import random
    rng = random.Random(1)
    two_pi = Fraction(62831853071795864769252867665590057683943387987502116419498891846156328125724, 10 ** 76)
    freq, place = [rng.uniform(2048, 4096) for _ in range(256)], [rng.randint(2 ** 23, 2 ** 24) for _ in range(150)]
    q = torch.zeros((150, 1, 512))
    q[:, :, :256] = 1                                                   # (1, 0): the cosine and the sine themselves
    got, _ = ps.Rotary([0] * 256, freq).forward(q.cuda(), None, torch.tensor(place, dtype=torch.float32)[:, None].cuda())
    got = got.double().cpu()[:, 0]
    turn = [[Fraction(p) * Fraction(f) / two_pi % 1 for f in freq] for p in place]
    want = torch.tensor([[float(t) for t in row] for row in turn], dtype=torch.float64) * (2 * math.pi)
    angle = torch.tensor(place, dtype=torch.float64)[:, None] * torch.tensor(freq, dtype=torch.float64)
    tol = 3 * 2.0 ** -53 * angle + 2.0 ** -22
    for part, exact in ((got[:, :256], torch.cos(want)), (got[:, 256:], torch.sin(want))):
        assert torch.all((part - exact).abs() <= tol), ((part - exact).abs() / angle).max() * 2 ** 52
