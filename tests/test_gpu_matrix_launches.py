"""What the matrix operators count as launched, and which of their kernels takes a call."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_1901_03040_b200 import qesgd                     # noqa: E402
from tests import gpu_helpers as G                          # noqa: E402


def _calls(ctx, rows, cols):
    """(name, call, launches) of every matrix operator, on buffers of their own."""
    x = torch.ones((rows, cols), device="cuda")
    codes, scales = qesgd.alloc_fp4(rows, cols, qesgd.FP4_NV, "cuda")
    codes_t, scales_t = qesgd.alloc_fp4(cols, rows, qesgd.FP4_NV, "cuda")
    for t in (codes, scales, codes_t, scales_t):
        t.zero_()
    e = torch.zeros(1, dtype=torch.int32, device="cuda")
    c, back = torch.zeros((rows, rows), device="cuda"), torch.zeros((rows, cols), device="cuda")
    o = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    work = torch.zeros(qesgd.orthogonalize_workspace(rows, cols), dtype=torch.uint8, device="cuda")
    need = work.numel()
    steps = 3
    return [
        ("exponent", lambda: ctx.qesgd_fp4_tensor_exponent(x, 0, rows, cols, cols, e), 1),
        ("quantize", lambda: ctx.qesgd_fp4_quantize(x, 0, rows, cols, cols, qesgd.FP4_NV, e, 0, 0, 0, 0, codes, scales, codes_t, scales_t), 1),
        ("dequantize", lambda: ctx.qesgd_fp4_dequantize(codes, scales, rows, cols, qesgd.FP4_NV, e, back, 0, cols), 1),
        ("product", lambda: ctx.qesgd_fp4_matmul(codes, scales, e, codes, scales, e, rows, rows, cols, qesgd.FP4_NV, c, 0, rows), 1),
        ("zeros", lambda: ctx.qesgd_fp4_matmul(None, None, None, None, None, None, rows, rows, 0, qesgd.FP4_NV, c, 0, rows), 1),
        ("orthogonalize", lambda: ctx.qesgd_orthogonalize(x, 0, rows, cols, cols, 1, 0, steps, o, cols, 0, work, need),
         1 if min(rows, cols) <= 128 else 2 + 3 * steps)]


@pytest.mark.parametrize("rows,cols", [(60, 100), (200, 300)])
def test_launches_are_counted_where_they_happen(rows, cols):
    """Each operator as it should be, and on a stream that takes no launch: one whose capture something has made
    invalid.  The refused call returns an error, counts nothing, and the next one runs."""
    cudart = ctypes.CDLL("libcudart.so.12")
    stream = torch.cuda.Stream()
    ctx = qesgd.Context(0, stream)
    calls = _calls(ctx, rows, cols)
    torch.cuda.synchronize()
    for name, call, launches in calls:
        before = ctx.qesgd_launch_count()
        call()
        assert ctx.qesgd_launch_count() - before == launches, name
    torch.cuda.synchronize()
    handle = ctypes.c_void_p(stream.cuda_stream)
    for name, call, launches in calls:
        before = ctx.qesgd_launch_count()
        graph = ctypes.c_void_p()
        assert cudart.cudaStreamBeginCapture(handle, 1) == 0
        try:
            assert cudart.cudaStreamSynchronize(handle) != 0           # not allowed in a capture, which it ends
            with pytest.raises(qesgd.QesgdError):
                call()
        finally:
            assert cudart.cudaStreamEndCapture(handle, ctypes.byref(graph)) != 0 and not graph.value
            cudart.cudaGetLastError()
        assert ctx.qesgd_launch_count() == before, name
        call()
        assert ctx.qesgd_launch_count() - before == launches, name
    assert ctx.qesgd_status() == 0
    ctx.close()


def test_a_product_of_more_tiles_than_a_grid_has_counts_nothing():
    ctx = G.ctx()
    some = torch.zeros(64, dtype=torch.uint8, device="cuda")
    before = ctx.qesgd_launch_count()
    side = qesgd.MAX_MATRIX_SIDE
    with pytest.raises(qesgd.QesgdError):
        ctx.qesgd_fp4_matmul(some, some, None, some, some, None, side, side, 32, qesgd.FP4_MX, some, qesgd.F32, side)
    assert ctx.qesgd_launch_count() == before and ctx.qesgd_status() == 0
