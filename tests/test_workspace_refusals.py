"""CPU-only: a caller's workspace that overlaps another buffer of the call is refused, whichever call takes it, and one that lies apart as far as the call
uses it is not (no kernel is launched: the library's entry points are replaced)."""
import ctypes as C

import pytest
import torch

import paper_2501_09253_amd as ps
from paper_2501_09253_amd import binding

NEED = 4096


class Library:
    """Entry points that return success; workspaces of NEED bytes."""

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_workspace"):
                args[-1]._obj.value = NEED
            return 0
        return call


@pytest.fixture
def alone(monkeypatch):
    library = Library()
    monkeypatch.setattr(binding, "lib", lambda: library)
    monkeypatch.setattr(binding, "_here", lambda *a: None)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    binding._prompt_desc.cache_clear()
    yield
    binding._prompt_desc.cache_clear()


def layer(kind, rows=8, K=64, N=32):
    op = kind.__new__(kind)
    op._h, op.K, op.N, op.dtype, op._dtype, op._row_bytes, op._bare = C.c_void_p(), K, N, ps.F32, torch.float32, NEED // rows, 0
    return op


def calls():
    """name: (call of a workspace and buffers, names and byte sizes of the buffers)"""
    f32, i32 = torch.float32, torch.int32
    rows, K, N = 8, 64, 32
    linear = dict(x=(f32, (rows, K)), res=(f32, (rows, N)), y=(f32, (rows, N)))
    attention = dict(q=(f32, (6, 4, 16)), k=(f32, (9, 2, 16)), v=(f32, (9, 2, 16)), cu_q=(i32, (3,)), cu_k=(i32, (3,)), out=(f32, (6, 4, 16)))
    paged = dict(q=(f32, (6, 4, 16)), cu_q=(i32, (3,)), key_len=(i32, (2,)), table=(i32, (2, 4)), out=(f32, (6, 4, 16)))
    store = ps.KV8.__new__(ps.KV8)
    store._h, store.places, store.kv_heads, store.head_dim = C.c_void_p(), 64, 2, 16
    return {
        "Linear8": (lambda ws, b: layer(ps.Linear8).forward(b["x"], res=b["res"], y=b["y"], workspace=ws), linear),
        "LinearF8": (lambda ws, b: layer(ps.LinearF8).forward(b["x"], res=b["res"], y=b["y"], workspace=ws), linear),
        "prompt_attention": (lambda ws, b: ps.prompt_attention(**b, workspace=ws), attention),
        "KV8.attention": (lambda ws, b: store.attention(page=8, workspace=ws, **b), paged),
    }


def laid_out(shapes, front=0):
    """An allocation with the buffers one after another from `front` on, and where they end."""
    arena, buffers, at = torch.zeros(200000, dtype=torch.uint8), {}, front
    for name, (dtype, shape) in shapes.items():
        n = torch.empty(shape, dtype=dtype).nbytes
        buffers[name] = arena[at:at + n].view(dtype).view(shape)
        at = -(-(at + n) // 16) * 16
    return arena, buffers, at


@pytest.mark.parametrize("name", list(calls()))
def test_a_workspace_over_a_buffer(alone, name):
    call, shapes = calls()[name]
    for over in shapes:
        arena, buffers, _ = laid_out(shapes, NEED)
        t, apart = buffers[over], torch.zeros(200000, dtype=torch.uint8)
        at = t.data_ptr() - arena.data_ptr()
        others = {k: (v if k == over else v.clone()) for k, v in buffers.items()}       # only `over` lies in the arena
        for begin in (at, at + t.nbytes - 4, at + 4 - NEED):                           # from its beginning, its last value, its first value
            with pytest.raises(ps.PserveError, match="workspace overlaps"):
                call(arena[begin:begin + NEED], others)
        call(apart[:NEED], others)


@pytest.mark.parametrize("name", list(calls()))
def test_a_workspace_beside_the_buffers(alone, name):
    call, shapes = calls()[name]
    arena, buffers, end = laid_out(shapes, NEED)
    call(arena[end:end + NEED], buffers)
    call(arena[:NEED], buffers)
    call(arena, buffers)                                    # larger than needed: what the call uses ends where the buffers begin
    call(None, buffers)
