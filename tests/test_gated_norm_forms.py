"""CPU: which form of the norms' kernel a call takes (host side of the dispatch, no kernel is launched), so that a change of the rule shows where it takes a
form's tests away."""
import pytest

import paper_2501_09253_amd as ps
from test_gpu_gated_norm_forms import CASES
from test_gpu_kv8 import CODE


@pytest.mark.parametrize("dtype,rows,C", list(CASES))
def test_cases_take_their_form(dtype, rows, C):
    assert tuple(ps.lib().pserve_test_gated_norm_form(CODE[dtype], rows, C, r8) for r8 in (0, 1)) == CASES[dtype, rows, C]


def test_every_form_has_its_cases():
    for dtype, forms in (("bf16", (81, 161, 321, 641, 642, 1, 2)), ("f32", (81, 161, 321, 641, 642, 1, 2, 4))):
        for even in (False, True):
            mine = [v for k, v in CASES.items() if k[0] == dtype and (k[2] % (8 if dtype == "bf16" else 4) == 0) == even]
            assert {v[0] for v in mine} == set(forms)
            assert {v[1] for v in mine} == set(f for f in forms if f >= (161 if dtype == "bf16" else 321) or f < 10)
