"""Rows in 8-bit floating point, bit for bit, and linear layers on them against the plain 64-bit form within the bound of tests/layer_oracle.py."""
import pytest
import torch

import layer_oracle as lo
import paper_2501_09253_amd as ps
from test_gpu_kv8 import CODE
from test_gpu_prompt_attention import DT, make

pytestmark = pytest.mark.gpu


def check(got, x, w, b, res):
    want, tol, size = lo.linear_f8(x, w, b, res, x.dtype)
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    ok = torch.isfinite(want)
    err = (got - want)[ok].abs()
    assert torch.all(err <= tol[ok]), (err / tol[ok]).max()
    if got.numel() >= 4096 and ok.all():
        # As a whole.  bf16: the output's rounding is even over a step of 2^-7 of a power of two (2^-7 / sqrt(12) of the value at most), with the
        # products' cut-off beside it: of eight products each loses 2^-14 of the largest on average, K / 8 times with either sign
        K = x.shape[1]
        share = {torch.bfloat16: 2.0 ** -7 / 12 ** 0.5 + 4e-4, torch.float32: (K / 16 + 32) * 4 * lo.U + 2 * lo.U}[x.dtype]
        assert (got - want).norm() <= share * want.norm(), ((got - want).norm() / want.norm()).item()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K", [(1, 1), (1, 128), (3, 5), (2, 129), (7, 640), (5, 1000), (33, 1027), (2, 4100), (300, 256)])
def test_rows_bit_for_bit(rows, K, dtype):
    x = make(rows, (rows, K), DT[dtype]) * torch.logspace(-30, 30, rows)[:, None].to(DT[dtype])
    x[0, :K // 2] = 0
    rows8 = ps.RowsF8(rows, K).write(x.cuda())
    code, scale, held = lo.f8_held(x)
    Kp, Sp = code.shape[1], -(-K // 512) * 4
    numbers, scales = rows8.buffer[:rows * Kp].view(rows, Kp).cpu(), rows8.buffer[rows * Kp:].view(Sp // 4, rows, 4).transpose(0, 1).reshape(rows, Sp).cpu()
    assert rows8.buffer.numel() == rows * (Kp + Sp)
    assert torch.equal(numbers & 127, code & 127) and torch.equal((numbers >= 128) & (code & 127 > 0), (code >= 128) & (code & 127 > 0))
    assert torch.equal(scales[:, :scale.shape[1]], scale) and torch.all(scales[:, scale.shape[1]:] == 127)
    for d in (ps.F32, ps.BF16):
        assert torch.equal(rows8.read(d).double().cpu(), held)


def test_halves_borders_and_extremes():
    """All halfway points of the format; blocks whose largest value stands at a power of two's border; the ends of fp32."""
    n = lo.f8_numbers()
    mid = (n[1:] + n[:-1]) / 2
    rows = [mid[:126], torch.cat([mid[100:], -n[:99]])]
    for peak in (448.0, 448.0000305, 449.0, 447.99997, 224.0, 3.4e38, 2.98e38, 2.99e38, 1.2e-28, 1e-35, 1e-45):
        rows.append(torch.cat([torch.tensor([peak], dtype=torch.float64), torch.linspace(-1, 1, 125, dtype=torch.float64) * peak]))
    x = torch.zeros((len(rows), 128))
    for i, r in enumerate(rows):
        x[i, 0], x[i, 1] = 448.0 if i < 2 else 0.0, 0.0
        x[i, 2:2 + len(r)] = r[:126].float()
    code, scale, held = lo.f8_held(x)
    rows8 = ps.RowsF8(*x.shape).write(x.cuda())
    assert torch.equal(rows8.read(ps.F32).double().cpu(), held)
    assert torch.equal(rows8.buffer[x.numel():].view(-1, 4)[:, :1].cpu(), scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_are_not_finite_and_rows_apart(dtype):
    wide = make(1, (6, 400), DT[dtype])
    x = wide[:, 3:303].clone()
    x[0, 5], x[1, 200], x[2, 299] = float("nan"), float("inf"), float("-inf")
    wide[:, 3:303] = x
    rows8 = ps.RowsF8(6, 300).write(wide.cuda()[:, 3:303])
    held, want = rows8.read(ps.F32).double().cpu(), lo.f8_held(x)[2]
    assert torch.equal(torch.isnan(held), torch.isnan(want)) and torch.equal(held.nan_to_num(), want.nan_to_num())
    assert torch.isnan(held[0, :128]).all() and torch.isfinite(held[0, 128:]).all() and torch.isnan(held[2, 256:]).all()


SHAPES = [(1, 64, 64), (1, 1, 1), (3, 77, 5), (12, 256, 512), (16, 4100, 130), (17, 128, 255), (33, 640, 1280), (64, 1000, 77), (130, 320, 264),
          (257, 129, 1000), (300, 2048, 640), (128, 128, 128), (129, 8200, 40), (700, 1536, 768), (1100, 384, 1152), (2, 16384, 33), (15, 513, 16), (20, 2300, 100), (31, 300, 6200), (16, 2049, 6145), (17, 5000, 50),
          (1300, 1100, 1030), (1281, 100, 1001), (5000, 700, 3400), (4200, 136, 4099),
          (40, 4100, 130), (250, 1027, 515), (100, 64, 4000), (17, 1500, 2050), (48, 2900, 33)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,N", SHAPES)
def test_against_64_bits(rows, K, N, dtype):
    x = make(1, (rows, K), DT[dtype]) * torch.logspace(-3, 3, rows)[:, None].to(DT[dtype])
    w, b, res = make(2, (K, N), DT[dtype], K ** -0.5), make(3, (N,), DT[dtype]), make(4, (rows, N), DT[dtype])
    for bias, r in ((b, None), (None, res), (b, res)):
        layer = ps.LinearF8(w.cuda(), None if bias is None else bias.cuda(), CODE[dtype])
        y = layer.forward(x.cuda(), res=None if r is None else r.cuda())
        check(y, x, w, bias, r)
    held = ps.RowsF8(rows, K).write(x.cuda())
    check(layer.forward(held, res=res.cuda()), x, w, b, res)


@pytest.mark.parametrize("rows,K,N", [(3000, 500, 3000), (3001, 130, 2999), (8000, 500, 4001), (9600, 1300, 4000), (16384, 300, 1000), (1, 700, 100000), (70000, 64, 96)])
def test_large_layers(rows, K, N):
    """Large tiles, several to a block, with and without edges; the reference's products on the GPU in 64 bits."""
    x, w = make(1, (rows, K), torch.bfloat16) * torch.logspace(-3, 3, rows)[:, None].to(torch.bfloat16), make(2, (K, N), torch.bfloat16, K ** -0.5)
    b, res = make(3, (N,), torch.bfloat16), make(4, (rows, N), torch.bfloat16)
    want, tol, _ = lo.linear_f8(x, w, b, res, torch.bfloat16, "cuda")
    layer = ps.LinearF8(w.cuda(), b.cuda(), ps.BF16)
    got = layer.forward(x.cuda(), res=res.cuda())
    assert torch.all((got.double() - want).abs() <= tol)
    rows8 = ps.RowsF8(rows, K).write(x.cuda())
    again = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda")
    for _ in range(3):                                                  # the same sums in the same order, whatever the blocks' pace
        layer.forward(rows8, res=res.cuda(), y=again)
        assert torch.equal(again, got)
    want, tol, _ = lo.linear_f8(x, w, b, None, torch.bfloat16, "cuda")
    assert torch.all((layer.forward(rows8).double() - want).abs() <= tol)


def test_offsets_past_32_bits():
    """2.5e9 outputs: the last rows are what they are in a call of their own (of as many rows as the tiles need)."""
    rows, K, N = 610000, 64, 4096
    x, w = torch.empty((rows, K), dtype=torch.bfloat16, device="cuda"), make(2, (K, N), torch.bfloat16, K ** -0.5).cuda()
    x.view(-1, 1000, K)[:] = make(1, (1000, K), torch.bfloat16).cuda()
    x[-5:] *= 2
    layer = ps.LinearF8(w, None, ps.BF16)
    got = layer.forward(x)
    for part in (slice(rows - 3000, rows), slice(rows // 2, rows // 2 + 3000)):
        assert torch.equal(got[part], layer.forward(x[part].clone()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,N", [(1, 96), (40, 96), (200, 96), (1500, 1500)])
def test_one_key_is_seen(rows, N, dtype):
    """Every value of K counts once and with its own block's scale: x picks single values out of W, block after block."""
    K = 700
    w = make(2, (K, N), DT[dtype]) * torch.logspace(-4, 4, K)[:, None].to(DT[dtype])
    layer = ps.LinearF8(w.cuda(), None, CODE[dtype])
    held = lo.f8_held(w.t().contiguous())[2].t()
    for k0 in range(0, K, 97):
        x = torch.zeros((rows, K), dtype=DT[dtype])
        for r in range(rows):
            x[r, (k0 + r) % K] = 1
        want = torch.stack([held[(k0 + r) % K] for r in range(rows)])
        got = layer.forward(x.cuda()).double().cpu()
        assert torch.all((got - want).abs() <= lo.HALF[DT[dtype]] * want.abs())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [5, 200, 20000])
def test_rows_apart_and_in_place(rows, dtype):
    K, N = 96, 160
    wide, w, b = make(1, (rows, K + 24), DT[dtype]), make(2, (K, N), DT[dtype]), make(3, (N,), DT[dtype])
    layer = ps.LinearF8(w.cuda(), b.cuda(), CODE[dtype])
    for off in (0, 8, 3):                                               # 3: rows off the 16-byte grid
        x = wide.cuda()[:, off:off + K]
        check(layer.forward(x), x.cpu(), w, b, None)
    y = make(4, (rows, N), DT[dtype])
    dev = y.cuda()
    layer.forward(x, res=dev, y=dev)
    check(dev, x.cpu(), w, b, y)
    odd = ps.LinearF8(w[:, :77].contiguous().cuda(), None, CODE[dtype])
    buf = torch.zeros(rows * 77 + 2, dtype=DT[dtype], device="cuda")
    odd.forward(x, y=buf[1:-1].view(rows, 77))                          # an output off the 16-byte grid
    check(buf[1:-1].view(rows, 77), x.cpu(), w[:, :77], None, None)
    assert buf[0] == 0 and buf[-1] == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [7, 150, 40000])
def test_zeros_extremes_and_what_is_not_finite(rows, dtype):
    x, w = make(1, (rows, 300), DT[dtype]), make(2, (300, 48), DT[dtype])
    x[0], w[:, 3] = 0, 0
    x[1] *= 1e-30
    x[2, 5], x[3, 299], w[7, 9], w[290, 11] = float("inf"), float("nan"), float("-inf"), float("nan")
    x[4] *= 1e30
    layer = ps.LinearF8(w.cuda(), None, CODE[dtype])
    check(layer.forward(x.cuda()), x, w, None, None)


def test_largest_numbers():
    """All numbers 448 at the largest K, with both signs."""
    K = 131072
    x = torch.full((2, K), 448.0)
    x[1] = -448
    w = torch.full((K, 3), 448.0)
    w[:, 1] = -448
    w[::2, 2] = -448
    layer = ps.LinearF8(w.cuda(), None, ps.F32)
    check(layer.forward(x.cuda()), x, w, None, None)
    layer = ps.LinearF8(w.bfloat16().cuda(), None, ps.BF16)
    check(layer.forward(x.bfloat16().cuda()), x.bfloat16(), w.bfloat16(), None, None)


@pytest.mark.parametrize("rows", [3, 150, 10000])
def test_graph_streams_and_workspace(rows):
    x, w, res = make(1, (rows, 320), torch.bfloat16).cuda(), make(2, (320, 192), torch.bfloat16).cuda(), make(3, (rows, 192), torch.bfloat16).cuda()
    layer = ps.LinearF8(w, None, ps.BF16)
    ws = torch.empty(layer.workspace_bytes(rows), dtype=torch.uint8, device="cuda")
    y = torch.empty_like(res)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = layer.forward(x, res=res, workspace=ws)
    side.synchronize()
    assert torch.equal(layer.forward(x, res=res), want)
    assert layer.forward(torch.empty((0, 320), dtype=torch.bfloat16, device="cuda")).shape == (0, 192)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(x, res=res, y=y, workspace=ws)
    for i in range(3):
        x.copy_(make(20 + i, (rows, 320), torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, layer.forward(x, res=res))
