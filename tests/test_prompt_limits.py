"""CPU-only: sizes that the prompt side asks for, and what its binding makes of arguments."""
import ctypes as C

import pytest
import torch

import paper_2501_09253_amd as ps
from paper_2501_09253_amd import binding
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


class _OnDevice(torch.Tensor):
    """A tensor of the host that says it is on device 0, for checks in front of any launch."""
    def get_device(self):
        return 0


def test_numbers_past_32_bits(monkeypatch):
    """Refused, not cut to their low half."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream", lambda: None)
    on = lambda t: t.as_subclass(_OnDevice)
    q, cu = on(torch.zeros(4, 2, 64, dtype=torch.bfloat16)), on(torch.zeros(2, dtype=torch.int32))
    key_len, table = on(torch.zeros(1, dtype=torch.int32)), on(torch.zeros(1, 4, dtype=torch.int32))
    for name in ("max_q", "max_k"):
        for value in (2 ** 31, 2 ** 32 + 5, -1):
            with pytest.raises(ps.PserveError, match=name):
                ps.prompt_attention(q, q, q, cu, **{name: value})
    store = ps.KV8.__new__(ps.KV8)
    store._h, store.places, store.kv_heads, store.head_dim = C.c_void_p(), 64, 2, 64
    for page in (2 ** 32 + 16, 2 ** 31, 0, -16):
        with pytest.raises(ps.PserveError, match="page"):
            store.attention(q, cu, key_len, table, page)
    for places, heads, dim, word in ((2 ** 64 + 64, 2, 64, "places"), (64, 2 ** 32 + 2, 64, "heads"), (64, 2, 2 ** 32 + 64, "head_dim")):
        with pytest.raises(ps.PserveError, match=word):
            ps.KV8(places, heads, dim)
