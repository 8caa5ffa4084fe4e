"""Arguments of the prompt side's binding that are not plain numbers."""
import numpy as np
import pytest
import torch

import paper_2501_09253_amd as ps
from test_gpu_prompt_attention import ints, make

pytestmark = pytest.mark.gpu


def test_a_scale_that_is_an_array_of_one():
    """The value it has at the call counts, not the one it had in an earlier call."""
    q = make(1, (40, 4, 64), torch.bfloat16).cuda()
    cu = ints([0, 40])
    store = ps.KV8(48, 4, 64)
    store.write(q, q, torch.arange(40, device="cuda"))
    for scale in (torch.tensor(0.1), np.full((), 0.1, dtype=np.float32)):
        for value in (0.1, 0.5, -0.3):
            scale[...] = value
            got = ps.prompt_attention(q, q, q, cu, scale=scale), store.attention(q, cu, ints([40]), ints([[0, 1, 2]]), 16, scale=scale)
            want = (ps.prompt_attention(q, q, q, cu, scale=float(scale)),
                    store.attention(q, cu, ints([40]), ints([[0, 1, 2]]), 16, scale=float(scale)))
            assert all(torch.equal(a, b) for a, b in zip(got, want))
