"""CPU-only: sizes that the prompt side asks for, and what its binding makes of arguments."""
import ctypes as C

import pytest

import paper_2501_09253_amd as ps
from test_prompt_refusals import desc


def workspace(d):
    need = C.c_size_t()
    assert ps.lib().pserve_prompt_attention_workspace(C.byref(d), C.byref(need)) == 0
    return need.value


@pytest.mark.parametrize("dtype", [ps.BF16, ps.F32])
@pytest.mark.parametrize("heads,kv_heads,dim", [(16, 4, 64), (32, 8, 128), (12, 12, 64), (8, 1, 80)])
@pytest.mark.parametrize("n,q_tokens,max_q,max_k", [(4, 1529, 640, 4095), (32, 32, 1, 8000), (1, 130, 130, 131072), (8, 616, 77, 77), (70, 800, 90, 2300), (2, 5000, 0, 0)])
def test_a_store_call_asks_for_no_packed_plan(n, q_tokens, max_q, max_k, heads, kv_heads, dim, dtype):
    """Where there are no packed keys the workspace is that of the call over the store, and no number of packed keys makes it smaller."""
    need = lambda k_tokens: workspace(desc(n=n, q_tokens=q_tokens, k_tokens=k_tokens, max_q=max_q, max_k=max_k, heads=heads, kv_heads=kv_heads, head_dim=dim, dtype=dtype))
    assert all(need(0) <= need(k) for k in (1, 100, q_tokens, 10 * q_tokens, 1 << 20))
