"""CPU: which form of the product an 8-bit floating-point layer takes (host side of the dispatch, no kernel is launched), so that a change of the rule
shows where it takes a form's tests away."""
import pytest

import paper_2501_09253_amd as ps
from test_gpu_linear_f8_forms import CASES, FROM_X, TILES_256

FORMS = {ps.F32: (1, 11, 12, 22, 64, 128), ps.BF16: (1, 11, 12, 22, 64, 128, 256)}


def form(dtype, rows, K, N, from_x=True, res=False):
    return ps.lib().pserve_test_linear_f8_form(dtype, rows, K, N, from_x, res)


@pytest.mark.parametrize("name", list(CASES))
def test_cases_take_their_form(name):
    dtype, want, rows, K, N = CASES[name]
    assert [form(dtype, rows, K, N, want == FROM_X, res) for res in (False, True)] == [want, want]


@pytest.mark.parametrize("dtype", [ps.F32, ps.BF16])
def test_every_form_has_its_cases(dtype):
    """Every form with more than four blocks of K (the scales' second word), whole lines of outputs and others, an edge in each direction."""
    for f in FORMS[dtype]:
        mine = [c[2:] for c in CASES.values() if c[:2] == (dtype, f)]
        line = 128 // (2 if dtype == ps.BF16 else 4)
        assert any(K > 512 for _, K, _ in mine) and any(K > 512 and K % 128 for _, K, _ in mine), f
        assert any(N % line == 0 for _, _, N in mine) and any(N % line for _, _, N in mine), f


def test_the_largest_tiles_come_out_uneven():
    """More tiles than blocks, in numbers that XCDs and blocks do not share evenly (blocks with one less begin later), and a whole number of rounds."""
    shares = []
    for dtype, f, rows, K, N in CASES.values():
        if f == TILES_256:
            total = -(-rows // 256) * -(-N // 256)
            shares += [(total * (x + 1) // 8 - total * x // 8) for x in range(8)]
    assert any(s > 32 and s % 32 for s in shares) and any(s and s % 32 == 0 for s in shares) and any(s < 32 for s in shares)


def test_sizes_of_any_kind_take_a_form():
    for dtype in (ps.F32, ps.BF16):
        for rows in (1, 16, 17, 100, 700, 5000, 40000, (1 << 26) - 1):
            for K in (1, 128, 129, 5000, 131072):
                for N in (1, 17, 4096, 50000, 1 << 24):
                    for res in (False, True):
                        assert form(dtype, rows, K, N, True, res) in FORMS[dtype] and form(dtype, rows, K, N, False, res) in FORMS[dtype][1:]
