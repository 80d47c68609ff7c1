"""The gated unit where a piece of 8 elements spans several rows: rows of x and w of 1 to 7 elements, and of [g | u] of 2 and 6, at numbers
of rows a little above a step's.  That no piece ends behind its operand is shown in test_glu_plan.py; here the sums have to be whole:
every row takes part, whichever way it is loaded.  Tolerances: test_gpu_glu's."""
import pytest

from test_gpu_glu import both_ways

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [31, 33, 64, 65, 70, 257, 263, 1027])
@pytest.mark.parametrize("H,F", [(1, 1), (1, 40), (2, 33), (3, 131), (4, 3), (5, 65), (7, 1), (40, 1), (129, 3)])
def test_rows_of_few_elements(T, H, F, dtype):
    both_ways(T, H, F, dtype, "gelu_erf", True)
