"""CPU: the largest layers that a call takes, and what lies beyond."""
import ctypes as C

import pytest

from paper_2306_11800_amd import api
from tests.test_answer_refusals import layer


@pytest.mark.parametrize("in_out", [0, 1])
def test_dimensions(in_out):
    """Up to 16 threads of a launch fall to an output (joining the parts of 4 rows) and up to 24 to an input (packing and
    turning 96 rows): 2^27 of either stay below the 2^32 threads that a launch may have."""
    lib, need = api.load_library(), C.c_uint64()
    for n_out, n_in, rc in ((1 << 27, 31, 0), (31, 1 << 27, 0), ((1 << 27) + 1, 4, -1), (4, (1 << 27) + 1, -1), (1 << 30, 3, -1),
                            (3, 1 << 30, -1)):
        c = layer()._c[1]
        c.n_out, c.n_in, c.in_out, c.weight.n = n_out, n_in, in_out, n_out * n_in
        assert lib.inshr_linear_bound(C.byref(c), 1, C.byref(need)) == rc, (n_out, n_in)
        assert lib.inshr_linear_grad_bound(C.byref(c), 1, 1, 1, C.byref(need)) == rc, (n_out, n_in)
