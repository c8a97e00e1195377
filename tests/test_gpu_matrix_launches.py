"""What the matrix operators count as launched, and which of their kernels takes a call."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from oracle import matrix_ref as ref                        # noqa: E402
from paper_1901_03040_b200 import qesgd                     # noqa: E402
from tests import gpu_helpers as G                          # noqa: E402
from tests.test_gpu_matrix_accuracy import ROUNDING, STEP, _exact, _off   # noqa: E402

FORMATS = [qesgd.FP4_MX, qesgd.FP4_NV]


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


# ---------------------------------------------------------------- which kernel ----
SHAPES = [(1, 64, 256, (1,)), (2, 128, 4000, (16,)), (1, 1000, 40, (4,)),
          (3, 129, 1000, (4, 8, 8, 8)), (1, 500, 500, (8, 8, 4, 8)), (6, 300, 2000, (2, 8, 1, 1)), (40, 300, 300, (1, 1, 1, 1)),
          (20, 450, 900, (16, 16, 16, 16)), (30, 500, 260, (1, 8, 16, 16)), (1, 1100, 2000, (2, 8, 0, 1)), (14, 600, 900, (1, 1, 0, 16)),
          (1, 2100, 2500, (16, 16, 0, 17)), (1, 2500, 2100, (16, 16, 0, 17)), (1, 4100, 4200, (16, 16, 0, 17))]


@pytest.mark.parametrize("batch,rows,cols,shapes", SHAPES)
def test_every_kernel_of_the_orthogonalisation(batch, rows, cols, shapes):
    """The one-kernel form by cluster sizes; else each product by single CTAs (1), ones that share a contraction (2, 4), narrow
    tiles (8), pairs of SMs (16) and pairs with the deep ring (17): stored by tiled copies and by plain stores (an odd ldo), and
    turned; several waves of pairs (4100 rows); from the first step's result to the fifth's."""
    whole = len(shapes) == 1
    for dtype, pad, back, steps in ((qesgd.F32, 0, 0, 5), (qesgd.BF16, 3, 1, 5), (qesgd.F16, 8, 8, 2), (qesgd.F32, 1, 0, 1)):
        if batch * rows * cols > 1 << 23 and (pad, steps) == (8, 2):
            continue
        g = torch.Generator(device="cuda").manual_seed(rows + pad)
        x = torch.randn((batch, rows, cols + pad), generator=g, device="cuda")
        x += torch.randn((batch, rows, 4), generator=g, device="cuda") @ torch.randn((batch, 4, cols + pad), generator=g, device="cuda")
        x = x.to({qesgd.F32: torch.float32, qesgd.BF16: torch.bfloat16, qesgd.F16: torch.float16}[dtype])
        out = torch.full((batch, rows, cols + back), 9.0, dtype=torch.bfloat16, device="cuda")
        need = qesgd.orthogonalize_workspace(rows, cols, batch)
        work = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")      # NaN in every type
        ctx = G.ctx()
        ctx.qesgd_orthogonalize(x, dtype, rows, cols, cols + pad, batch, x.stride(0), steps, out, cols + back, out.stride(0), work, need)
        plan = ctx.qesgd_debug_matrix_plan()
        if whole:
            assert plan[:2] == (qesgd.MATRIX_ORTHO_WHOLE, shapes[0])
        else:   # with few steps no update takes one term alone
            only = (*shapes[:3], 0) if shapes[2] and steps <= 3 else shapes
            assert plan[:5] == (qesgd.MATRIX_ORTHO_PRODUCTS, *only)
        for i in range(batch):
            off = _off(out[i:i + 1, :, :cols], _exact(x[i:i + 1, :, :cols], steps))[0]
            assert off <= float(np.hypot(ROUNDING, np.sqrt(steps) * STEP)), (dtype, pad, steps, i, off)
        assert (out[:, :, cols:] == 9.0).all() and (work[need:] == 0xFF).all()
        assert ctx.qesgd_status() == 0


@pytest.mark.parametrize("M,N,K,kind", [(2304, 2500, 3000, "pairs"), (1900, 2101, 1500, "pairs"), (300, 520, 700, "singles"), (2100, 2400, 300, "singles"),
                                        (64, 1000, 9000, "shared"), (3, 300, 4096, "shared")])
@pytest.mark.parametrize("fmt", FORMATS)
def test_every_kernel_of_the_product(fmt, M, N, K, kind):
    """Each output type, stored and added to, with and without the tensors' exponents (NV), aligned rows of C and odd ones, by
    pairs of SMs, single CTAs and clusters that share a contraction.  Values up to 1.5 and scales of 1/2, 1 and 2: sums are multiples
    of 2^-4 below 9 * 9000 < 2^17, exact in any order."""
    g = np.random.default_rng(K)
    held = []
    for rows in (M, N):
        codes = g.integers(0, 4, (rows, K), dtype=np.uint8) + 8 * g.integers(0, 2, (rows, K), dtype=np.uint8)
        pick = np.array([126, 127, 128] if fmt == qesgd.FP4_MX else [0x30, 0x38, 0x40], dtype=np.uint8)
        byte = pick[g.integers(0, 3, (rows, -(-K // ref.BLOCK[fmt])))]
        held.append((torch.from_numpy(ref.values(codes, byte, fmt)).cuda(), G.dev(ref.pack(codes)), G.dev(ref.tiles(byte))))
    (a, ca, sa), (b, cb, sb) = held
    want = a @ b.T
    types = {qesgd.F32: torch.float32, qesgd.BF16: torch.bfloat16, qesgd.F16: torch.float16}
    exponents = [None] if fmt == qesgd.FP4_MX else [None, (-3, 1), (90, -93), (-100, -40), (100, 20), (200, -300)]
    for e in exponents:
        power = 1.0 if e is None else 2.0 ** sum(min(max(t, -126), 126) for t in e)
        ta, tb = (None, None) if e is None else torch.tensor(e, dtype=torch.int32, device="cuda").split(1)
        for dtype, pad, acc in ((qesgd.F32, 0, 0), (qesgd.F32, 3, 1), (qesgd.BF16, 0, 1), (qesgd.BF16, 1, 0), (qesgd.F16, 0, 1), (qesgd.F16, 2, 0)):
            c = torch.randint(-8, 9, (M, N + pad), generator=torch.Generator().manual_seed(N)).to(types[dtype]).cuda()
            before = c.clone()
            ctx = G.ctx()
            ctx.qesgd_fp4_matmul(ca, sa, ta, cb, sb, tb, M, N, K, fmt, c, dtype, N + pad, acc)
            plan = ctx.qesgd_debug_matrix_plan()
            assert plan[0] == (qesgd.MATRIX_PRODUCT_PAIRS if kind == "pairs" else qesgd.MATRIX_PRODUCT_SINGLES)
            assert (plan[1] > 1) == (kind != "singles")
            # scaled exactly (2^-140 times a multiple of 2^-4 is one of fp32's subnormals; 2^120 times some sums is infinite in 32 bits),
            # added in 32 bits, rounded to C's type
            full = (power * want + (before[:, :N].double() if acc else 0.0)).float().to(types[dtype])
            assert torch.equal(c[:, :N], full), (e, dtype, pad, acc)
            assert torch.equal(c[:, N:], before[:, N:])
        assert ctx.qesgd_status() == 0


@pytest.mark.parametrize("rows,cols,tile", [(130, 38000, 64), (4000, 2500, 64), (257, 1000, 32), (33, 31, 32)])
@pytest.mark.parametrize("dtype", [qesgd.F32, qesgd.BF16, qesgd.F16])
@pytest.mark.parametrize("scaled", [False, True])
def test_both_tiles_of_the_row_quantiser(scaled, dtype, rows, cols, tile):
    """Tiles of 64 rows (more of them than run at once) and of 32, with and without the tensor's exponent, nearest and drawn."""
    g = torch.Generator().manual_seed(rows)
    x = torch.randn((rows, cols + 1), generator=g) * 1e-3
    x[torch.rand((rows, cols + 1), generator=g) < 0.02] *= 30.0
    x = x.to({qesgd.F32: torch.float32, qesgd.BF16: torch.bfloat16, qesgd.F16: torch.float16}[dtype]).cuda()
    v = x[:, :cols].cpu().double().numpy()
    ctx, fmt, t, e = G.ctx(), qesgd.FP4_NV if scaled else qesgd.FP4_MX, 0, None
    if scaled:
        e = torch.zeros(1, dtype=torch.int32, device="cuda")
        ctx.qesgd_fp4_tensor_exponent(x, dtype, rows, cols, cols + 1, e)
        t = ref.tensor_exponent(v)
        assert int(e) == t
    for seed in (None, 9):
        codes, scales = qesgd.alloc_fp4(rows, cols, fmt, "cuda")
        codes.fill_(0xAB), scales.fill_(0xAB)
        ctx.qesgd_fp4_quantize(x, dtype, rows, cols, cols + 1, fmt, e, 0 if seed is None else 1, seed or 0, 4, 5, codes, scales)
        assert ctx.qesgd_debug_matrix_plan()[:2] == (qesgd.MATRIX_QUANTIZE_ROWS, tile)
        want_codes, want_bytes, _ = ref.quantize(v, fmt, t, seed, 4, 5)
        assert (scales.cpu().numpy() == ref.tiles(want_bytes)).all()
        assert (codes.cpu().numpy() == ref.pack(want_codes)).all()
    assert ctx.qesgd_status() == 0
