"""CPU-only: which numbers of rows an 8-bit floating-point layer needs a workspace for, as the binding finds it when a layer is made and as the library says for
each number (host side only; creating the layer is replaced)."""
import ctypes as C

import pytest
import torch

import paper_2501_09253_amd as ps
from paper_2501_09253_amd import binding


class Library:
    """The library, with a layer that is an image of the fields that its host side reads (K, N; rounded up; dtype); counts the questions."""

    def __init__(self, K, N, dtype):
        self.asked = 0
        self.image = (C.c_int64 * 64)(K | N << 32, -(-K // 128) * 128 | -(-N // 256) * 256 << 32, dtype)

    def pserve_linear_f8_create(self, *args):
        args[-1]._obj.value = C.addressof(self.image)
        return 0

    def pserve_linear_f8_workspace(self, layer, rows, need):
        self.asked += 1
        return ps.lib().pserve_linear_f8_workspace(layer, rows, need)

    def pserve_linear_f8_free(self, layer):
        pass


@pytest.mark.parametrize("dtype", [ps.F32, ps.BF16])
@pytest.mark.parametrize("K,N", [(1, 1), (64, 16), (100, 40), (1024, 1), (1280, 640), (2048, 256), (2049, 256), (6144, 100), (6145, 100), (131072, 8), (300, 70000)])
def test_rows_that_need_a_workspace(monkeypatch, K, N, dtype):
    library = Library(K, N, dtype)
    monkeypatch.setattr(binding, "_here", lambda *a: None)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    with monkeypatch.context() as m:
        m.setattr(binding, "lib", lambda: library)
        layer = ps.LinearF8(torch.zeros((K, N), dtype=torch.float32 if dtype == ps.F32 else torch.bfloat16), None, dtype)
        try:
            assert library.asked <= 20                                  # a search, not a walk over all numbers of rows
            for rows in list(range(0, 700)) + list(range(16300, 16500)) + [1000, 5000, 40000, (1 << 26) - 1]:
                assert layer.workspace_bytes(rows) == (0 if rows <= layer._bare else rows * layer._row_bytes), rows
        finally:
            layer.close()
