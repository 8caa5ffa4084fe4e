"""CPU-only: the error bounds of the prompt attention's tests notice what they are there for, planted in the plain form."""
import pytest
import torch

import prompt_exact as pe


def with_weights(q, k, v, scale, change):
    """Attention of one head over all keys whose normalised weights go through `change`."""
    p = torch.softmax((q @ k.t()) * scale, 1)
    return (change(p) @ v).bfloat16().double()


@pytest.mark.parametrize("Lk,D", [(100, 64), (300, 128), (3000, 128), (9000, 64)])
def test_a_missing_key_and_a_rounded_weight(Lk, D):
    g = torch.Generator().manual_seed(Lk)
    q, k, v = (torch.randn(n, 1, D, generator=g, dtype=torch.float64).bfloat16().double() for n in (64, Lk, Lk))
    out, bound, spread, size = pe.attention(q, k, v, D ** -0.5, False)
    run = lambda change: with_weights(q[:, 0], k[:, 0], v[:, 0], D ** -0.5, change).unsqueeze(1)
    once = lambda p: p.float().bfloat16().double()
    two = lambda p: once(p) + once(p - once(p))
    tight = pe.tolerance(out, bound, size, torch.bfloat16, D, Lk, pe.TWO_PIECES)
    loose = pe.tolerance(out, bound, size, torch.bfloat16, D, Lk, pe.ONE_PIECE)
    norm = lambda piece: pe.norm_bound(out, bound, spread, size, torch.bfloat16, D, Lk, piece)
    good, near = run(two) - out, run(once) - out
    assert torch.all(good.abs() <= tight) and good.norm() <= norm(pe.TWO_PIECES)
    assert torch.all(near.abs() <= loose) and near.norm() <= norm(pe.ONE_PIECE)
    if Lk <= 300:                                                       # one bf16 number where two are promised
        assert not torch.all(near.abs() <= tight)
    for at in (0, Lk // 2, Lk - 1):                                     # a key left out, a key counted twice
        for times in (0.0, 2.0):
            lost = run(lambda p: two(p * torch.where(torch.arange(Lk) == at, times, 1.0))) - out
            assert lost.norm() > norm(pe.TWO_PIECES)
