"""CPU-only: what the prompt-side entry points refuse (no kernel is launched, no pointer is read)."""
import ctypes as C

import pytest
import torch

import paper_2501_09253_amd as ps
from paper_2501_09253_amd import binding

P = 4096                        # an aligned address that nothing reads


def desc(**change):
    d = binding._PromptDesc()
    d.n, d.heads, d.kv_heads, d.head_dim, d.dtype, d.causal, d.scale = 2, 8, 2, 64, ps.BF16, 1, 0.125
    d.q_tokens, d.k_tokens = 10, 10
    d.q_stride[:], d.o_stride[:] = (512, 64), (512, 64)
    d.k_stride[:], d.v_stride[:] = (128, 64), (128, 64)
    for k, v in change.items():
        if isinstance(v, tuple):
            getattr(d, k)[:] = v
        else:
            setattr(d, k, v)
    return d


def refused(status, word):
    assert status == -1 and word in ps.lib().pserve_last_error().decode(), (status, ps.lib().pserve_last_error())


@pytest.mark.parametrize("change,word", [
    (dict(n=0), "n > 0"), (dict(heads=7), "heads"), (dict(kv_heads=0), "heads"), (dict(heads=8192), "4096"), (dict(head_dim=72), "head_dim"),
    (dict(head_dim=144), "head_dim"), (dict(head_dim=0), "head_dim"), (dict(dtype=2), "dtype"), (dict(scale=float("nan")), "scale"),
    (dict(q_tokens=-1), "sizes"), (dict(q_tokens=2 ** 31), "sizes"), (dict(max_k=-1), "sizes"), (dict(k_tokens=-1), "sizes"),
    (dict(q_stride=(515, 64)), "stride"), (dict(o_stride=(-512, 64)), "stride"), (dict(k_stride=(128, 4)), "stride"), (dict(v_stride=(1 << 28, 64)), "stride")])
def test_prompt_attention_refuses(change, word):
    L = ps.lib()
    refused(L.pserve_prompt_attention(C.byref(desc(**change)), P, P, P, P, P, None, 0, P, None), word)


def test_prompt_attention_buffers():
    L, d = ps.lib(), desc()
    refused(L.pserve_prompt_attention(None, P, P, P, P, P, None, 0, P, None), "NULL")
    for i in range(6):
        args = [P, P, P, P, P, P]
        args[i] = None
        refused(L.pserve_prompt_attention(C.byref(d), *args[:5], None, 0, args[5], None), "NULL")
    for i in (0, 1, 2, 5):
        args = [P, P, P, P, P, P]
        args[i] = P + 2
        refused(L.pserve_prompt_attention(C.byref(d), *args[:5], None, 0, args[5], None), "aligned")
    need = C.c_size_t()
    long = desc(max_k=100000)
    assert L.pserve_prompt_attention_workspace(C.byref(long), C.byref(need)) == 0 and need.value > 0
    refused(L.pserve_prompt_attention(C.byref(long), P, P, P, P, P, P, need.value - 1, P, None), "workspace")
    refused(L.pserve_prompt_attention(C.byref(long), P, P, P, P, P, None, need.value, P, None), "workspace")
    refused(L.pserve_prompt_attention_workspace(C.byref(long), None), "NULL")
    assert L.pserve_prompt_attention(C.byref(desc(q_tokens=0)), None, None, None, None, None, None, 0, None, None) == 0


def test_store_and_layer_refuse():
    L, out = ps.lib(), C.c_void_p()
    for places, heads, dim in ((0, 8, 64), (2 ** 31, 8, 64), (64, 0, 64), (64, 8, 24), (64, 8, 144), (64, 8, 0)):
        assert L.pserve_kv8_create(places, heads, dim, None, C.byref(out)) == -1 and not out.value
    refused(L.pserve_kv8_create(64, 8, 64, None, None), "NULL")
    s = (C.c_int64 * 2)(512, 64)
    refused(L.pserve_kv8_write(None, P, P, 1, s, s, P, 4, None), "NULL")
    refused(L.pserve_kv8_read(None, P, 4, 1, P, P, None), "NULL")
    refused(L.pserve_kv8_attention(None, C.byref(desc()), P, P, P, P, 4, 16, None, 0, P, None), "NULL")
    for K, N, dtype, w in ((0, 8, 1, P), (8, 0, 1, P), (131073, 8, 1, P), (8, 8, 5, P), (8, 8, 1, None)):
        assert L.pserve_linear8_create(K, N, dtype, w, None, None, C.byref(out)) == -1 and not out.value
    refused(L.pserve_linear8_create(8, 8, 1, P, None, None, None), "NULL")
    refused(L.pserve_linear8_forward(None, P, 8, 4, None, P, 1000, P, None), "NULL")
    refused(L.pserve_linear8_workspace(None, 4, C.byref(C.c_size_t())), "NULL")


def test_binding_refuses_tensors_that_are_not_on_the_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    q, cu = torch.zeros(4, 2, 64), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ps.PserveError, match="device"):
        ps.prompt_attention(q, q, q, cu)
    with pytest.raises(ps.PserveError, match="device"):
        ps.Linear8(torch.zeros(8, 8), None, ps.F32)


def test_scales_that_overflow_in_the_kernel():
    refused(ps.lib().pserve_prompt_attention(C.byref(desc(scale=3e38)), P, P, P, P, P, None, 0, P, None), "scale")


def test_more_rows_than_a_launch_has_threads():
    """Refused by size alone, before any launch: the objects here are images of the fields that the checks read."""
    L = ps.lib()
    store = (C.c_int64 * 64)()
    store[0], store[1] = 1000, 4096 | 128 << 32                         # places; heads, head_dim
    s = (C.c_int64 * 2)(4096 * 128, 128)
    for rows in (1 << 16, 1 << 28, 1 << 40):
        refused(L.pserve_kv8_write(store, P, P, 1, s, s, P, rows, None), "rows")
        refused(L.pserve_kv8_read(store, P, rows, 1, P, P, None), "rows")
    layer = (C.c_int64 * 64)()
    layer[0], layer[1], layer[2] = 1 | 1 << 32, 128 | 256 << 32, 1      # K, N; rounded up; dtype
    need = C.c_size_t()
    assert L.pserve_linear8_workspace(layer, (1 << 26) - 1, C.byref(need)) == 0 and need.value == ((1 << 26) - 1) * 132
    refused(L.pserve_linear8_workspace(layer, 1 << 26, C.byref(need)), "rows")
    refused(L.pserve_linear8_forward(layer, P, 1, 1 << 26, None, P, 1 << 40, P, None), "rows")


def test_too_many_tiles():
    """2^31 tokens less one of 4096 heads: more 16-row tiles than 31 bits number, more wide ones than a launch has blocks."""
    L = ps.lib()
    for dtype in (ps.BF16, ps.F32):
        d = desc(q_tokens=2 ** 31 - 1, heads=4096, kv_heads=4096, dtype=dtype, max_q=2 ** 20, max_k=2 ** 20)
        refused(L.pserve_prompt_attention(C.byref(d), P, P, P, P, P, P, 1 << 60, P, None), "tiles")
