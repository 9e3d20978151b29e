"""tgrad_codes_gradient and the sizes of its scratch: what is refused, before the device is looked at.  No kernel runs here."""
import ctypes as C

import pytest

from paper_2501_02379_amd import tgrad as T
from test_block8_abi import BAD, BAD_CODES, BAD_MATRICES, codes, mat

OPS = [op + more for op in (T.TGRAD_CODES_GRAD_INPUT, T.TGRAD_CODES_GRAD_WEIGHT) for more in (0, T.TGRAD_CODES_UNALIGNED, T.TGRAD_CODES_UNROUNDED, 12)]


@pytest.mark.parametrize("op", OPS)
def test_refusals(op):
    call = T.load().tgrad_codes_gradient
    weight = op % 4 == T.TGRAD_CODES_GRAD_WEIGHT
    c, out = (codes(8, 50), mat(100, 50)) if weight else (codes(100, 50), mat(8, 50))
    for change in BAD_MATRICES:
        assert call(op, mat(**change), c, out, 256, None) == BAD
        assert call(op, mat(), c, mat(**change), 256, None) == BAD
    for change in BAD_CODES:
        assert call(op, mat(), codes(**change), out, 256, None) == BAD
    assert call(op, mat(), codes(9, 50), out, 256, None) == BAD
    assert call(op, mat(), c, mat(7, 50), 256, None) == BAD
    assert call(op, mat(), c, mat(100 if weight else 8, 50, dtype=T.TGRAD_F16), 256, None) == BAD
    assert call(op, mat(80, 99), codes(80, 50) if weight else codes(99, 50), mat(99, 50) if weight else mat(80, 50), None, None) == BAD      # odd rows need scratch


@pytest.mark.parametrize("op", [-1, 0, 1, 4, 5, 8, 9, 13, 16, 18, 1 << 20])
def test_other_ops_are_refused(op):
    n = C.c_size_t(0)
    assert T.load().tgrad_codes_gradient(op, mat(), codes(100, 50), mat(8, 50), 256, None) == BAD
    if op not in (0, 1):
        assert T.load().tgrad_codes_query_size(op, 8, 50, 100, C.byref(n)) == BAD


def test_unrounded_values_need_no_more_scratch():
    n, m = C.c_size_t(0), C.c_size_t(0)
    for op in OPS:
        for sizes in ((1, 1, 1), (700, 300, 200), (131072, 512, 768), (8192, 8192, 8192)):
            assert T.load().tgrad_codes_query_size(op, *sizes, C.byref(n)) == T.TGRAD_OK
            assert T.load().tgrad_codes_query_size(op | T.TGRAD_CODES_UNROUNDED, *sizes, C.byref(m)) == T.TGRAD_OK and n.value == m.value
