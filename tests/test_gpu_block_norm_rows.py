"""The norms' backward pass where a workgroup goes from row to row: the next row's loads ahead, sums in two places of LDS in turn, a row of the gate kept until
its last row, column sums in registers.  Formulas and tolerances are those of test_gpu_block_norm.py.

Rows of 256, 600, 2560, 4100, 8192 columns are held by every kind of workgroup that there is, those of 16400 by several; each size has three rows a chunk or more
with the number of chunks that the sizes allow.
"""
import ctypes as C

import pytest
import torch

from paper_2501_02379_amd import norms, tgrad as T
from test_gpu_block_norm import check, make

pytestmark = pytest.mark.gpu

SIZES = [(8200, 256), (2050, 600), (1030, 2560), (520, 4100), (520, 8192), (260, 16400)]
KINDS = [("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("f32", "f32")]
# each token, two to a chunk's three, more than a chunk, some chunks with a shorter last one, all tokens
SHARED = [1, 2, 4, 100, 1 << 40]


@pytest.mark.parametrize("centered", [False, True])
@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("size", range(len(SIZES)))
def test_several_rows_a_workgroup(size, kind, centered):
    rows, cols = SIZES[size]
    check(rows, cols, *KINDS[kind], SHARED[(size + 2 * kind + centered) % len(SHARED)], centered, seed=size)


@pytest.mark.parametrize("shared", SHARED)
@pytest.mark.parametrize("rows,cols", [(1030, 2560), (260, 16400)])
def test_gates_of_every_share(rows, cols, shared):
    check(rows, cols, "bf16", "bf16", shared, shared % 4 == 0, pad=3)


@pytest.mark.parametrize("parts", [{"with_post": False}, {"with_gate": False}, {"with_pre": False}, {"with_dx": False}])
@pytest.mark.parametrize("rows,cols", [(1030, 2560), (260, 16400)])
def test_parts_of_several_rows(rows, cols, parts):
    check(rows, cols, "f32", "f16", 2, True, **parts)


@pytest.mark.parametrize("stream,dtype", [("bf16", "bf16"), ("f32", "f16")])
@pytest.mark.parametrize("rows,cols", [(2050, 600), (520, 8192), (260, 16400)])
def test_the_gradient_goes_where_it_came_from(rows, cols, stream, dtype):
    """dx may be dx_out."""
    s = make(rows, cols, stream, dtype, 4)
    args = {"post_weight": s["post"], "gate": s["gate"], "rows_per_gate": 4, "scale": 0.5, "pre_weight": s["pre"]}
    f = norms.tgrad_block_norm(s["x"], s["block"], **args)
    want = norms.tgrad_block_norm_backward(s["dx"], s["dh"], f.x, s["block"], stats=f.stats, **args)
    got = [t.clone() if t is s["dx"] else torch.empty_like(t) for t in (s["dx"], want.dblock, want.dgate, want.dpost, want.dpre)]
    codes = {torch.float32: T.TGRAD_F32, torch.bfloat16: T.TGRAD_BF16, torch.float16: T.TGRAD_F16}
    mat = lambda t: C.byref(T.tgrad_matrix(t.data_ptr(), rows, cols, t.stride(0), codes[t.dtype]))  # noqa: E731
    n = C.c_size_t(0)
    assert T.load().tgrad_block_norm_query_size(rows, cols, 4, C.byref(n)) == T.TGRAD_OK
    ws = torch.empty(n.value, dtype=torch.uint8, device=s["x"].device)
    d = T.tgrad_block(s["post"].data_ptr(), s["pre"].data_ptr(), s["gate"].data_ptr(), s["gate"].stride(0), 4, T.TGRAD_F32, 0.5, 1.0, 0)
    assert T.load().tgrad_block_norm_backward(C.byref(d), mat(got[0]), mat(s["dh"]), mat(f.x), mat(s["block"]), f.stats.data_ptr(), mat(got[0]), mat(got[1]),
                                              got[2].data_ptr(), got[3].data_ptr(), got[4].data_ptr(), ws.data_ptr(), torch.cuda.current_stream().cuda_stream) == T.TGRAD_OK
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, (want.dx, want.dblock, want.dgate, want.dpost, want.dpre)))
