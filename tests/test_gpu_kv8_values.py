"""What the 8-bit store gives back, bit for bit, and the places that it has."""
import pytest
import torch

import paper_2501_09253_amd as ps
import prompt_oracle as po
from test_gpu_prompt_attention import make

pytestmark = pytest.mark.gpu


def nearest_bf16(x):
    """64-bit numbers in bf16's normal range to the nearest of bf16, halves to even, without a step between."""
    assert torch.all((x == 0) | (x.abs() >= 2.0 ** -126))
    u = x.view(torch.int64)
    u = (u + (1 << 44) - 1 + ((u >> 45) & 1)) & ~((1 << 45) - 1)       # 53 bits to 8; the sign is a bit of its own
    return u.view(torch.float64)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,dim", [(8, 128), (12, 64), (3, 80)])
def test_values_are_rounded_once(heads, dim, dtype):
    """Whole number times fp32 scale has up to 31 bits: of the fp32 rows 3 to 55 values lie so close to the middle of two bf16 numbers that
    their fp32 product is the middle."""
    rows = 4000
    k, v = make(1, (rows, heads, dim), dtype), make(2, (rows, heads, dim), dtype, 30.0)
    store, at = ps.KV8(rows, heads, dim), torch.arange(rows, device="cuda")
    store.write(k.cuda(), v.cuda(), at)
    for x, half, whole in zip((k, v), store.read(at, ps.BF16), store.read(at, ps.F32)):
        q, s = po.steps(x)
        exact = q * s.float().double()                                  # 31 bits: exact in 64
        near = nearest_bf16(exact)
        assert (near != exact.float().bfloat16().double()).sum() >= (3 if dtype == torch.float32 else 0)
        assert torch.equal(half.cpu().double(), near)
        assert torch.equal(whole.cpu(), exact.float())
