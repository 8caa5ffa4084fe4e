"""Workspaces of exactly the bytes that were asked for."""
import pytest
import torch

import paper_2501_09253_amd as ps
from paper_2501_09253_amd import binding
from test_gpu_kv8 import check_cached, paged
from test_gpu_prompt_attention import check, ints, make, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lq,lk,heads,kv_heads,dim", [([60, 12, 90], [900, 70, 1300], 8, 2, 64), ([1, 1, 3], [40, 2000, 700], 8, 2, 128), ([70], [2500], 4, 4, 80)])
def test_exactly_what_is_needed(lq, lk, heads, kv_heads, dim, dtype):
    q, k, v = (make(i, (sum(n), h, dim), dtype) for i, n, h in ((1, lq, heads), (2, lk, kv_heads), (3, lk, kv_heads)))
    cu, ck = ints(starts(lq)), ints(starts(lk))
    table, places, total = paged(lk, 16, 4)
    store = ps.KV8(total, kv_heads, dim)
    store.write(k.cuda(), v.cuda(), places)
    dev = [t.cuda() for t in (q, k, v)]

    def need(k_tokens):
        none = (0, 0) if k_tokens == 0 else dev[1].stride()
        return binding._prompt_desc(len(lq), heads, kv_heads, dim, ps.BF16 if dtype == torch.bfloat16 else ps.F32, True, None, max(lq), max(lk),
                                    sum(lq), k_tokens, dev[0].stride(), none, none, dev[0].stride())[1]

    def over(room):
        return store.attention(dev[0], cu, ints(lk), table, 16, max_q=max(lq), max_k=max(lk), workspace=room)

    behind = 4096
    for bytes_, call, test in ((need(0), over, lambda o: check_cached(o, q, k, v, lq, lk)),
                               (need(sum(lk)), lambda room: ps.prompt_attention(*dev, cu, ck, max_q=max(lq), max_k=max(lk), workspace=room),
                                lambda o: check(o, q, k, v, lq, lk))):
        assert bytes_ > 0
        room = torch.full((bytes_ + behind,), 77, dtype=torch.uint8, device="cuda")
        test(call(room[:bytes_]))
        assert torch.all(room[bytes_:] == 77)
    with pytest.raises(ps.PserveError, match="workspace"):              # the store's plan takes all that was asked for
        over(torch.empty(need(0) - 1, dtype=torch.uint8, device="cuda"))
