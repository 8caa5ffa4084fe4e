"""Every form of the norms' kernel (threads of a row, chunks of a thread; whole chunks or not) against the plain 64-bit form, with h and with 8-bit rows, rows of
several requests and of none.  Each case checks which form it takes."""
import pytest
import torch

import layer_oracle as lo
import paper_2501_09253_amd as ps
from test_gpu_gated_norm import gpu, inputs, near, near8
from test_gpu_kv8 import CODE
from test_gpu_prompt_attention import ints

pytestmark = pytest.mark.gpu

# dtype, rows, C: form with h, with 8-bit rows
CASES = {
    ("bf16", 700, 64): (81, 161), ("bf16", 700, 61): (81, 161), ("bf16", 700, 128): (161, 161), ("bf16", 700, 125): (161, 161),
    ("bf16", 300, 256): (321, 321), ("bf16", 300, 131): (321, 321), ("bf16", 300, 512): (641, 641), ("bf16", 300, 389): (641, 641),
    ("bf16", 9001, 640): (642, 642), ("bf16", 9001, 517): (642, 642), ("bf16", 8192, 1024): (642, 642), ("bf16", 8195, 1021): (642, 642),
    ("bf16", 101, 640): (1, 1), ("bf16", 101, 517): (1, 1), ("bf16", 31, 4096): (1, 1), ("bf16", 31, 4091): (1, 1),
    ("bf16", 11, 4104): (2, 2), ("bf16", 11, 4099): (2, 2), ("bf16", 11, 16384): (2, 2), ("bf16", 11, 16383): (2, 2),
    ("f32", 700, 32): (81, 321), ("f32", 700, 29): (81, 321), ("f32", 700, 64): (161, 321), ("f32", 700, 61): (161, 321),
    ("f32", 300, 128): (321, 321), ("f32", 300, 126): (321, 321), ("f32", 300, 256): (641, 641), ("f32", 300, 131): (641, 641),
    ("f32", 9001, 320): (642, 642), ("f32", 9001, 261): (642, 642), ("f32", 8192, 512): (642, 642), ("f32", 8195, 509): (642, 642),
    ("f32", 101, 320): (1, 1), ("f32", 101, 261): (1, 1), ("f32", 31, 2048): (1, 1), ("f32", 31, 2045): (1, 1),
    ("f32", 11, 2052): (2, 2), ("f32", 11, 2050): (2, 2), ("f32", 11, 8192): (2, 2), ("f32", 11, 8191): (2, 2),
    ("f32", 11, 8196): (4, 4), ("f32", 11, 8195): (4, 4), ("f32", 11, 16384): (4, 4), ("f32", 11, 16383): (4, 4), ("f32", 11, 4099): (2, 2),
}


class Part:
    """The values that a part of the rows holds."""

    def __init__(self, rows8, part):
        self.rows8, self.part = rows8, part

    def read(self, dtype):
        return self.rows8.read(dtype)[self.part]


@pytest.mark.parametrize("dtype,rows,C", list(CASES))
def test_form(dtype, rows, C):
    assert tuple(ps.lib().pserve_test_gated_norm_form(CODE[dtype], rows, C, r8) for r8 in (0, 1)) == CASES[dtype, rows, C]
    t = inputs(rows, C, dtype, 4)
    cu = [1, 1 + rows // 3, 1 + rows // 3, rows - 4, rows - 2]           # a row of no request in front, an empty request, two rows of none behind
    request = torch.cat([torch.full((cu[i + 1] - cu[i],), i) for i in range(4)])
    mine = slice(cu[0], cu[-1])
    kinds = dict(post="layer", pre="rms", skip_scale=0.8, branch_scale=1.5)
    wy, wh = lo.gated_norm(**dict(t, x=t["x"][mine], f=t["f"][mine]), **kinds, request=request)
    y, h = (torch.full((rows, C), 7.0, dtype=t["x"].dtype, device="cuda") for _ in range(2))
    ps.gated_norm(**gpu(t), **kinds, cu_rows=ints(cu), y=y, h=h)
    near(y[mine], wy, dtype)
    near(h[mine], wh, dtype)
    for out in (y, h):
        assert torch.all(out[:cu[0]] == 7) and torch.all(out[cu[-1]:] == 7)
    rows8 = ps.RowsF8(rows, C)
    rows8.buffer.fill_(33)
    again = torch.full_like(y, 7.0)
    ps.gated_norm(**gpu(t), **kinds, cu_rows=ints(cu), y=again, rows8=rows8)
    assert torch.equal(again[mine], y[mine]) or CASES[dtype, rows, C][0] != CASES[dtype, rows, C][1]      # (other forms sum in another order)
    near(again[mine], wy, dtype)
    near8(Part(rows8, mine), wh)
    width = -(-C // 128) * 128
    numbers = rows8.buffer[:rows * width].view(rows, width)
    assert torch.all(numbers[:cu[0]] == 33) and torch.all(numbers[cu[-1]:] == 33) and torch.all(numbers[mine, C:] & 127 == 0)
    scales = rows8.buffer[rows * width:].view(-1, rows, 4).transpose(0, 1)
    assert torch.all(scales[:cu[0]] == 33) and torch.all(scales[cu[-1]:] == 33)
    assert torch.all(scales[mine].reshape(cu[-1] - cu[0], -1)[:, width // 128:] == 127)
