"""What the sums of the 8-bit floating-point layers lose, without the output's rounding in front of it: the residual takes the result away, so what is
left is rounded 2^-9 times as finely."""
import pytest
import torch

import layer_oracle as lo
import paper_2501_09253_amd as ps
from test_gpu_kv8 import CODE
from test_gpu_prompt_attention import DT, make

pytestmark = pytest.mark.gpu


# few rows rounded on the way in; few rows; the tiles
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,N", [(12, 4096, 512), (40, 4100, 130), (16, 8192, 1024), (333, 640, 1920), (700, 1536, 768), (2048, 2048, 640), (5000, 700, 3400), (3000, 3000, 3000)])
def test_what_the_sums_lose(rows, K, N, dtype):
    dt = DT[dtype]
    x, w, b = make(1, (rows, K), dt), make(2, (K, N), dt, K ** -0.5), make(3, (N,), dt)
    whole = lo.linear_f8(x, w, b, None, dt, "cuda")[0]
    res = -whole.to(dt)
    want, tol, _ = lo.linear_f8(x, w, b, res.cpu(), dt, "cuda")
    layer = ps.LinearF8(w.cuda(), b.cuda(), CODE[dtype])
    got = layer.forward(x.cuda(), res=res)
    off = got.double() - want
    assert torch.all(off.abs() <= tol), (off.abs() / tol).max().item()
    # As a whole.  bf16: of eight products each loses less than 2^-13 of the largest, whose square is at most the eight squares' sum on average, with either
    # sign: K losses of 2^-13 sqrt(8) of a product's size beside a result of sqrt(K) of it.  Sums in fp32: a step of 2 U of a partial sum at most for each of
    # the K / 16 + 32 additions, with either sign.  What is left is at most half a step of the result, and its rounding as much of that again
    sums = 2 * lo.U * (K / 16 + 32) ** 0.5
    share = (8 ** 0.5 * 2.0 ** -13 if dtype == "bf16" else 0.0) + sums + 2 * lo.U + lo.HALF[dt] ** 2
    assert off.norm() <= share * whole.norm(), (off.norm() / whole.norm()).item()
    for _ in range(3):                                                  # the same bits every time
        assert torch.equal(layer.forward(x.cuda(), res=res), got)
    held = ps.RowsF8(rows, K).write(x.cuda())
    off = layer.forward(held, res=res).double() - want                  # (other kernels, where rows are few)
    assert torch.all(off.abs() <= tol) and off.norm() <= share * whole.norm()
