"""What the entry points of a block in 8 bits refuse, checked before they look at the device.  No kernel runs here."""
import ctypes as C

import pytest

from paper_2501_02379_amd import tgrad as T

BAD = T.TGRAD_ERR_INVALID_ARG


def mat(rows=8, cols=100, stride=None, dtype=T.TGRAD_BF16, data=4096):
    return C.byref(T.tgrad_matrix(data, rows, cols, cols if stride is None else stride, dtype))


def codes(rows=8, cols=100, stride=None, group=0, data=4096, scale=8192):
    return C.byref(T.tgrad_codes(data, scale, rows, cols, cols if stride is None else stride, group))


BAD_MATRICES = [{"data": None}, {"data": 4097}, {"rows": -1}, {"rows": 1 << 31}, {"cols": 0}, {"cols": 1 << 31}, {"stride": 99}, {"stride": 1 << 62},
                {"dtype": T.TGRAD_C64}, {"dtype": 5}, {"dtype": T.TGRAD_F32, "data": 4098}]
BAD_CODES = [{"data": None}, {"scale": None}, {"scale": 8194}, {"rows": -1}, {"rows": 1 << 31}, {"cols": 0}, {"stride": 99}, {"stride": 1 << 62},
             {"group": 16}, {"group": -1}, {"group": 48}, {"group": 1024}]


@pytest.mark.parametrize("change", BAD_MATRICES)
def test_bad_matrices_are_refused(change):
    lib = T.load()
    assert lib.tgrad_quantize(mat(**change), codes(), None) == BAD
    assert lib.tgrad_dequantize(codes(), mat(**change), None) == BAD
    assert lib.tgrad_codes_matmul(codes(), codes(100), mat(**change), 256, None) == BAD
    assert lib.tgrad_codes_linear(mat(**change), codes(100), None, mat(), 256, None) == BAD
    assert lib.tgrad_codes_linear(mat(), codes(100), None, mat(**change), 256, None) == BAD
    assert lib.tgrad_codes_grad_input(mat(**change), codes(100, 50), mat(8, 50), 256, None) == BAD
    assert lib.tgrad_codes_grad_weight(mat(**change), codes(8, 50), mat(100, 50), 256, None) == BAD
    assert lib.tgrad_activation(mat(**change), None, 0, mat(), None, None, None, None) == BAD
    assert lib.tgrad_activation(mat(), mat(**change), 0, mat(), None, None, None, None) == BAD
    assert lib.tgrad_activation(mat(), None, 0, mat(**change), None, None, None, None) == BAD
    assert lib.tgrad_activation_backward(mat(**change), codes(group=32), None, 0, mat(), None, None) == BAD
    d = C.byref(T.tgrad_block(256, 512, None, 0, 1, T.TGRAD_F32, 1.0, 1e-6, 0))
    assert lib.tgrad_block_norm(d, mat(**change), mat(), mat(), mat(), None, None, None) == BAD
    assert lib.tgrad_block_norm(d, mat(), mat(), mat(**change), mat(), None, None, None) == BAD
    assert lib.tgrad_block_norm_backward(d, mat(), mat(**change), mat(), mat(), 256, mat(), mat(), None, 256, 512, 1024, None) == BAD
    assert lib.tgrad_block_norm_backward(d, mat(), mat(), mat(), mat(), 256, mat(**change), mat(), None, 256, 512, 1024, None) == BAD


@pytest.mark.parametrize("change", BAD_CODES)
def test_bad_codes_are_refused(change):
    lib = T.load()
    assert lib.tgrad_quantize(mat(), codes(**change), None) == BAD
    assert lib.tgrad_dequantize(codes(**change), mat(), None) == BAD
    assert lib.tgrad_codes_matmul(codes(**change), codes(100), mat(), 256, None) == BAD
    assert lib.tgrad_codes_matmul(codes(100), codes(**change), mat(100, 8), 256, None) == BAD
    assert lib.tgrad_codes_linear(mat(), codes(100), codes(**change), mat(), 256, None) == BAD
    assert lib.tgrad_codes_grad_weight(mat(), codes(**change), mat(100, 100), 256, None) == BAD
    assert lib.tgrad_activation_backward(mat(), codes(**change), None, 0, mat(), None, None) == BAD


def test_sizes_have_to_go_together():
    lib = T.load()
    ok32 = codes(group=32)
    f32 = T.TGRAD_F32
    assert lib.tgrad_quantize(mat(8, 100), codes(8, 99), None) == BAD
    assert lib.tgrad_dequantize(codes(7), mat(), None) == BAD
    assert lib.tgrad_codes_matmul(codes(), codes(40, 99), mat(8, 40), 256, None) == BAD
    assert lib.tgrad_codes_matmul(codes(), codes(40), mat(8, 41), 256, None) == BAD
    assert lib.tgrad_codes_matmul(ok32, codes(40), mat(8, 40), 256, None) == BAD          # one scale a row in both
    assert lib.tgrad_codes_matmul(codes(), codes(40, group=32), mat(8, 40), 256, None) == BAD
    for ws in (264, None):                                                                # 40 tokens need scratch
        assert lib.tgrad_codes_matmul(codes(40, 4096), codes(40, 4096), mat(40, 40), ws, None) == BAD
        assert lib.tgrad_codes_linear(mat(20), codes(40), None, mat(20, 40), ws, None) == BAD
        assert lib.tgrad_codes_grad_weight(mat(80, 99), codes(80, 50), mat(99, 50), ws, None) == BAD      # and so does dy with odd rows
    long = 131073
    assert lib.tgrad_codes_matmul(codes(1, long), codes(1, long), mat(1, 1), 256, None) == T.TGRAD_ERR_UNSUPPORTED
    assert lib.tgrad_codes_linear(mat(1, long), codes(1, long), None, mat(1, 1), 256, None) == T.TGRAD_ERR_UNSUPPORTED
    assert lib.tgrad_codes_linear(mat(), codes(40), codes(7), mat(8, 40), 256, None) == BAD
    assert lib.tgrad_codes_linear(mat(), codes(40), ok32, mat(8, 40), 256, None) == BAD
    assert lib.tgrad_codes_grad_input(mat(), codes(99, 50), mat(8, 50), 256, None) == BAD
    assert lib.tgrad_codes_grad_input(mat(), codes(100, 50), mat(8, 50, dtype=T.TGRAD_F16), 256, None) == BAD
    assert lib.tgrad_codes_grad_input(mat(dtype=f32, data=4096), codes(100, 50), mat(8, 50), 256, None) == BAD
    assert lib.tgrad_codes_grad_weight(mat(), codes(9, 50), mat(100, 50), 256, None) == BAD
    assert lib.tgrad_activation(mat(), mat(dtype=f32), 0, mat(), None, None, None, None) == BAD
    assert lib.tgrad_activation(mat(), None, 2, mat(), None, None, None, None) == BAD
    assert lib.tgrad_activation(mat(), None, 0, None, None, ok32, None, None) == BAD       # no result
    assert lib.tgrad_activation(mat(), None, 0, mat(), codes(), ok32, None, None) == BAD   # two of them
    assert lib.tgrad_activation(mat(), None, 0, mat(), None, codes(), None, None) == BAD   # a checkpoint is in groups
    assert lib.tgrad_activation(mat(), mat(), 0, mat(), None, ok32, None, None) == BAD     # a gate without its checkpoint
    assert lib.tgrad_activation(mat(), None, 0, mat(), None, ok32, ok32, None) == BAD
    assert lib.tgrad_activation(mat(), None, 0, None, ok32, None, None, None) == BAD       # the next product wants one scale a row
    assert lib.tgrad_activation_backward(mat(), ok32, ok32, 0, mat(), None, None) == BAD
    assert lib.tgrad_activation_backward(mat(), ok32, None, 0, mat(dtype=f32), None, None) == BAD
    assert lib.tgrad_activation_backward(mat(), ok32, None, -1, mat(), None, None) == BAD


def test_norm_arguments_are_checked():
    lib = T.load()
    f32, f16 = T.TGRAD_F32, T.TGRAD_F16
    nan, inf = float("nan"), float("inf")

    def desc(post=256, pre=512, gate=None, stride=100, shared=1, wt=f32, scale=1.0, eps=1e-6, centered=0):
        return T.tgrad_block(post, pre, gate, stride, shared, wt, scale, eps, centered)

    def forward(d=None, x=mat(), block=mat(), out=mat(), h=mat(), h8=None, stats=None):
        return lib.tgrad_block_norm(C.byref(d or desc()), x, block, out, h, h8, stats, None)

    def backward(d=None, up=mat(), dh=mat(), x=mat(), block=mat(), stats=256, dx=mat(), db=mat(), dgate=None, dpost=256, dpre=512, ws=1024):
        return lib.tgrad_block_norm_backward(C.byref(d or desc()), up, dh, x, block, stats, dx, db, dgate, dpost, dpre, ws, None)

    wide = 32769
    for d in (desc(wt=0), desc(wt=5), desc(scale=nan), desc(scale=inf), desc(eps=0.0), desc(eps=-1.0), desc(eps=nan), desc(eps=inf), desc(centered=2),
              desc(post=258), desc(pre=513), desc(gate=4097), desc(gate=4096, shared=0), desc(gate=4096, stride=99)):
        assert forward(d) == BAD and backward(d, dgate=4096 if d.gate else None) == BAD
    for change in ({"out": None}, {"block": None}, {"h": None}, {"h8": codes()}, {"h": None, "h8": codes(group=32)}, {"h": mat(7)}, {"h": mat(dtype=f16)},
                   {"block": mat(dtype=f16)}, {"block": mat(8, 99)}, {"out": mat(dtype=f32)}, {"stats": 8}, {"d": desc(pre=None)},
                   {"block": None, "out": None}, {"block": None, "out": None, "d": desc(post=None, gate=4096)},
                   {"block": None, "out": None, "h": None, "d": desc(post=None, pre=None)}, {"x": mat(dtype=f16), "out": mat(dtype=f16)}):
        assert forward(**change) == BAD
    for change in ({"dh": None}, {"dh": mat(dtype=f16)}, {"up": mat(dtype=f16)}, {"up": mat(9)}, {"x": mat(9)}, {"block": None}, {"db": None},
                   {"db": mat(dtype=f16)}, {"dx": mat(dtype=f32)}, {"stats": None}, {"stats": 264}, {"dgate": 4096}, {"d": desc(gate=4096)}, {"dpost": None},
                   {"dpre": None}, {"dpost": 258}, {"ws": None}, {"ws": 1032}, {"d": desc(post=None)}, {"d": desc(pre=None)},
                   {"dx": mat(stride=108), "up": mat(stride=104)}):
        assert backward(**change) == BAD
    w = mat(1, wide)
    assert forward(x=w, block=w, out=w, h=w) == T.TGRAD_ERR_UNSUPPORTED
    assert backward(up=w, dh=w, x=w, block=w, dx=w, db=w) == T.TGRAD_ERR_UNSUPPORTED


def test_sizes_of_scratch():
    lib = T.load()
    n = C.c_size_t(0)
    got = []
    for tokens in (0, 1, 1000, 100000):
        assert lib.tgrad_codes_query_size(T.TGRAD_CODES_LINEAR, tokens, 4096, 4096, C.byref(n)) == T.TGRAD_OK
        assert n.value % 256 == 0 and n.value >= (tokens * 4096 if tokens > 4 else 0)
        got.append(n.value)
    assert got == sorted(got)
    for op in range(4):
        for sizes in ((0, 33, 55), (77, 33, 0), (0, 33, 0), (1, 1, 1), (1, 1 << 20, 1 << 20)):
            assert lib.tgrad_codes_query_size(op, *sizes, C.byref(n)) == T.TGRAD_OK and n.value % 256 == 0
        assert lib.tgrad_codes_query_size(op, 77, 33, 55, C.byref(n)) == T.TGRAD_OK and n.value % 256 == 0
    for args in ((-1, 1, 1, 1), (4, 1, 1, 1), (0, -1, 1, 1), (0, 1, 0, 1), (0, 1, 1, -1), (0, 1 << 31, 1, 1), (0, 1, 1 << 31, 1)):
        assert lib.tgrad_codes_query_size(*args, C.byref(n)) == BAD
    assert lib.tgrad_codes_query_size(0, 1, 1, 1, None) == BAD
    assert lib.tgrad_block_norm_query_size(1000, 4096, 1, C.byref(n)) == T.TGRAD_OK and n.value % 256 == 0 and n.value >= 2 * 4096 * 4
    assert lib.tgrad_block_norm_query_size(0, 5, 7, C.byref(n)) == T.TGRAD_OK and n.value >= 256
    assert lib.tgrad_block_norm_query_size(1, wide := 32769, 1, C.byref(n)) == T.TGRAD_ERR_UNSUPPORTED and wide
    for args in ((-1, 1, 1), (1, 0, 1), (1, 1, 0)):
        assert lib.tgrad_block_norm_query_size(*args, C.byref(n)) == BAD
    assert lib.tgrad_block_norm_query_size(1, 1, 1, None) == BAD
