"""Every form of the product of an 8-bit floating-point layer against the plain 64-bit form, at sizes that the rule gives it: more blocks of K than a word
of scales holds, whole lines of outputs and others, edges, tiles in numbers that blocks do not share evenly.  Each case checks which form it takes."""
import pytest
import torch

import layer_oracle as lo
import paper_2501_09253_amd as ps
from test_gpu_prompt_attention import make

pytestmark = pytest.mark.gpu

FROM_X, FEW_16_16, FEW_16_32, FEW_32_32, TILES_64, TILES_128, TILES_256 = 1, 11, 12, 22, 64, 128, 256
# dtype, form, rows, K, N
CASES = {
    "bf16_from_x": (ps.BF16, FROM_X, 37, 1280, 640),
    "bf16_from_x_edges": (ps.BF16, FROM_X, 19, 1700, 1111),
    "bf16_16_16": (ps.BF16, FEW_16_16, 33, 8200, 192),
    "bf16_16_16_edges": (ps.BF16, FEW_16_16, 2, 16300, 333),
    "bf16_16_32": (ps.BF16, FEW_16_32, 16, 2049, 6144),
    "bf16_16_32_edges": (ps.BF16, FEW_16_32, 17, 1500, 2050),
    "bf16_32_32": (ps.BF16, FEW_32_32, 300, 2048, 640),
    "bf16_32_32_edges": (ps.BF16, FEW_32_32, 250, 1027, 515),
    "bf16_64": (ps.BF16, TILES_64, 700, 1536, 768),
    "bf16_64_edges": (ps.BF16, TILES_64, 1300, 1100, 1030),
    "bf16_128": (ps.BF16, TILES_128, 9600, 1300, 4032),
    "bf16_128_edges": (ps.BF16, TILES_128, 5001, 700, 3401),
    "bf16_256_largest": (ps.BF16, TILES_256, 12544, 1536, 6144),
    "bf16_256_feed": (ps.BF16, TILES_256, 12544, 1536, 4608),
    "bf16_256_edges": (ps.BF16, TILES_256, 7901, 1347, 4001),
    "bf16_256_five_blocks": (ps.BF16, TILES_256, 7901, 600, 4001),
    "bf16_256_whole_lines": (ps.BF16, TILES_256, 7901, 1100, 4032),
    "bf16_256_four_blocks": (ps.BF16, TILES_256, 8192, 512, 4096),
    "bf16_256_one_round": (ps.BF16, TILES_256, 3000, 3000, 3000),
    "f32_from_x": (ps.F32, FROM_X, 37, 1280, 256),
    "f32_from_x_edges": (ps.F32, FROM_X, 19, 900, 1111),
    "f32_16_16": (ps.F32, FEW_16_16, 33, 8200, 192),
    "f32_16_16_edges": (ps.F32, FEW_16_16, 20, 2300, 101),
    "f32_16_32": (ps.F32, FEW_16_32, 16, 2049, 6144),
    "f32_16_32_edges": (ps.F32, FEW_16_32, 17, 1500, 2050),
    "f32_32_32": (ps.F32, FEW_32_32, 300, 2048, 640),
    "f32_32_32_edges": (ps.F32, FEW_32_32, 250, 1027, 515),
    "f32_64": (ps.F32, TILES_64, 700, 1536, 768),
    "f32_64_edges": (ps.F32, TILES_64, 1300, 1100, 1030),
    "f32_128": (ps.F32, TILES_128, 5000, 700, 3424),
    "f32_128_edges": (ps.F32, TILES_128, 5001, 1300, 3401),
}


@pytest.mark.parametrize("name", list(CASES))
def test_form(name):
    dtype, form, rows, K, N = CASES[name]
    dt = torch.bfloat16 if dtype == ps.BF16 else torch.float32
    for res in (False, True):
        assert ps.lib().pserve_test_linear_f8_form(dtype, rows, K, N, form == FROM_X, res) == form
    x, w = make(1, (rows, K), dt) * torch.logspace(-3, 3, rows)[:, None].to(dt), make(2, (K, N), dt, K ** -0.5)
    x = x * torch.logspace(0, 2, -(-K // 128))[torch.arange(K) // 128].to(dt)          # (blocks of a row with scales of their own)
    b, res = make(3, (N,), dt), make(4, (rows, N), dt)
    layer, dx, dres = ps.LinearF8(w.cuda(), b.cuda(), dtype), x.cuda(), res.cuda()
    source = dx if form == FROM_X else ps.RowsF8(rows, K).write(dx)
    plain, tol, _ = lo.linear_f8(x, w, b, None, dt, "cuda")
    got = layer.forward(source)
    assert torch.all((got.double() - plain).abs() <= tol)
    del tol
    want, tol, _ = lo.linear_f8(x, w, b, res, dt, "cuda")
    del plain
    got = layer.forward(source, res=dres)
    assert torch.all((got.double() - want).abs() <= tol)
    again = torch.full((rows + 2, N), 7.0, dtype=dt, device="cuda")
    again[1:-1] = dres
    layer.forward(source, res=again[1:-1], y=again[1:-1])              # in place of the residual; the same bits
    assert torch.equal(again[1:-1], got) and torch.all(again[0] == 7) and torch.all(again[-1] == 7)
