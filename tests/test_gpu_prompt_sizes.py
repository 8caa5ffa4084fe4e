"""The largest calls that the 8-bit store and the 8-bit layers take: launches of 2^24 blocks and more, and where a second line of blocks begins."""
import pytest
import torch

import paper_2501_09253_amd as ps
import prompt_oracle as po
from test_gpu_kv8 import same
from test_gpu_linear8 import check
from test_gpu_prompt_attention import make

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory_back():
    yield
    torch.cuda.empty_cache()


# 9 heads of 80: a block for each row
@pytest.mark.parametrize("rows", [(1 << 20) + 5, 3 * (1 << 20) - 1, ((1 << 28) - 1) // 9])
def test_rows_written(rows):
    heads, dim, places = 9, 80, 500
    base = make(1, (1 << 16,), torch.bfloat16).cuda().repeat((8 * rows + 8000 + heads * dim) // (1 << 16) + 1)
    k = base.as_strided((rows, heads, dim), (8, dim, 1))                # a row begins 16 bytes behind the one before it
    v = base.as_strided((rows, heads, dim), (8, dim, 1), 8000)
    last = {0: 3, 1: rows // 2, 2: rows - 1, 7: rows - 2, 499: (1 << 20) + 1, 44: 1 << 20}
    at = torch.full((rows,), -1, dtype=torch.int64, device="cuda")
    at[:64] = 7                                                         # taken again by a later row
    at[torch.tensor(sorted(last.values()), device="cuda")] = torch.tensor([p for p, _ in sorted(last.items(), key=lambda x: x[1])], device="cuda")
    store = ps.KV8(places, heads, dim)
    for _ in range(2):
        store.write(k, v, at)
        got = store.read(torch.arange(places, device="cuda"), ps.F32)
        rest = [p for p in range(places) if p not in last]
        for t, x in zip(got, (k, v)):
            same(t[list(last)], po.held(x[list(last.values())].cpu()), torch.float32)
            assert torch.all(t[rest] == 0)


@pytest.mark.parametrize("rows", [(1 << 24) + 5, (1 << 28) - 1])
def test_rows_read(rows):
    places, dim = 1000, 80
    if torch.cuda.mem_get_info()[0] < 4 * rows * dim + 8 * rows + (8 << 30):
        pytest.skip("not enough free memory for the outputs")
    k, v = make(1, (places, 1, dim), torch.bfloat16).cuda(), make(2, (places, 1, dim), torch.bfloat16).cuda()
    store = ps.KV8(places, 1, dim)
    store.write(k, v, torch.arange(places, device="cuda"))
    at = torch.arange(rows, device="cuda").remainder_(places + 3)       # three of them out of range
    few = store.read(torch.arange(places + 3, device="cuda"), ps.BF16)
    got = store.read(at, ps.BF16)
    for t, x in zip(got, few):
        whole = rows // (places + 3) * (places + 3)
        for part in t[:whole].view(-1, places + 3, 1, dim).split(20000):
            assert torch.all(part == x)
        assert torch.equal(t[whole:], x[:rows - whole])


@pytest.mark.parametrize("rows", [(1 << 22) + 1, (1 << 26) - 1])
def test_rows_of_a_layer(rows):
    K, N = 8, 8
    x, w = make(1, (4096, K), torch.bfloat16).cuda(), make(2, (K, N), torch.bfloat16)
    many = x.repeat(rows // 4096 + 1, 1)[:rows]
    layer = ps.Linear8(w.cuda(), None, ps.BF16)
    few = layer.forward(x)
    check(few, x.cpu(), w, None, None)
    got = layer.forward(many)
    whole = rows // 4096 * 4096
    assert torch.all(got[:whole].view(-1, 4096, N) == few) and torch.equal(got[whole:], few[:rows - whole])
