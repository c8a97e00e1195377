"""The matrix operators at the ends of their sizes: one row or column of 65536, batches of 4096, rows of nearly 2^31 elements; and at addresses and
strides that only the element type aligns."""
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


@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 65536), (1, 65536, 1), (2, 2, 65536), (1, 5000, 3), (1, 65536, 130), (1, 300, 65536), (4096, 1, 1),
                                             (4096, 3, 40), (300, 129, 130)])
def test_orthogonalize_at_the_ends_of_its_sizes(batch, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn((batch, rows, cols), generator=g, device="cuda")
    need = qesgd.orthogonalize_workspace(rows, cols, batch)
    work = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full((batch, rows, cols + 1), 9.0, dtype=torch.bfloat16, device="cuda")
    G.ctx().qesgd_orthogonalize(x, qesgd.F32, rows, cols, cols, batch, rows * cols, 5, out, cols + 1, rows * (cols + 1), work, need)
    want = _exact(x)
    off = _off(out[:, :, :cols], want)
    # single elements' rounding where there are few: 2^-8 at most
    assert max(off) <= (np.hypot(ROUNDING, np.sqrt(5.0) * STEP) if min(rows, cols) >= 16 else 2.0 ** -8 + np.sqrt(5.0) * STEP), max(off)
    assert (out[:, :, cols:] == 9.0).all() and (work[need:] == 0xFF).all()
    assert G.ctx().qesgd_status() == 0


@pytest.mark.parametrize("rows,cols", [(20, 72), (200, 304)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_addresses_that_only_the_element_type_aligns(dtype, rows, cols):
    """x and every output one element behind a 16-byte boundary, rows of a multiple of 16 bytes; what lies around stays."""
    kind = {torch.float32: qesgd.F32, torch.bfloat16: qesgd.BF16, torch.float16: qesgd.F16}[dtype]
    ctx = G.ctx()
    n = rows * cols
    g = torch.Generator().manual_seed(rows)
    buf = torch.randn(n + 16, generator=g).to(dtype).cuda()
    x = buf[1:1 + n].view(rows, cols)
    v = x.cpu().double().numpy()
    for fmt in (qesgd.FP4_MX, qesgd.FP4_NV):
        e = None if fmt == qesgd.FP4_MX else torch.zeros(1, dtype=torch.int32, device="cuda")
        if e is not None:
            ctx.qesgd_fp4_tensor_exponent(x, kind, rows, cols, cols, e)
            assert int(e) == ref.tensor_exponent(v)
        t = 0 if e is None else int(e)
        held, held_t = qesgd.alloc_fp4(rows, cols, fmt, "cuda"), qesgd.alloc_fp4(cols, rows, fmt, "cuda")
        ctx.qesgd_fp4_quantize(x, kind, rows, cols, cols, fmt, e, 1, 3, 1, 2, *held, *held_t)
        for (codes, scales), m in ((held, v), (held_t, v.T)):
            want_codes, want_bytes, _ = ref.quantize(m, fmt, t, 3, 1, 2)
            assert (scales.cpu().numpy() == ref.tiles(want_bytes)).all() and (codes.cpu().numpy() == ref.pack(want_codes)).all()
        want_codes, want_bytes, _ = ref.quantize(v, fmt, t, 3, 1, 2)
        back = torch.full((n + 16,), 7.0, dtype=dtype, device="cuda")
        ctx.qesgd_fp4_dequantize(*held, rows, cols, fmt, e, back[1:], kind, cols)
        values = ref.values(want_codes, want_bytes, fmt, t)
        assert torch.equal(back[1:1 + n].view(rows, cols).cpu(), torch.from_numpy(values).to(dtype))
        assert back[0] == 7.0 and (back[1 + n:] == 7.0).all()
        size = rows * rows
        c = torch.full((size + 16,), 7.0, dtype=dtype, device="cuda")
        near = torch.zeros((rows, rows), dtype=dtype, device="cuda")
        for out, acc in ((c[1:], 0), (c[1:], 1), (near, 0), (near, 1)):
            ctx.qesgd_fp4_matmul(*held, e, *held, e, rows, rows, cols, fmt, out, kind, rows, acc)
        assert torch.equal(c[1:1 + size].view(rows, rows), near) and c[0] == 7.0 and (c[1 + size:] == 7.0).all()
    need = qesgd.orthogonalize_workspace(rows, cols)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    o = torch.full((n + 16,), 7.0, dtype=torch.bfloat16, device="cuda")
    near = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    ctx.qesgd_orthogonalize(x, kind, rows, cols, cols, 1, 0, 5, o[1:], cols, 0, work, need)
    ctx.qesgd_orthogonalize(x.clone(), kind, rows, cols, cols, 1, 0, 5, near, cols, 0, work, need)
    torch.cuda.synchronize()
    assert torch.equal(o[1:1 + n].view(rows, cols), near) and o[0] == 7.0 and (o[1 + n:] == 7.0).all()
    assert ctx.qesgd_status() == 0


@pytest.mark.parametrize("fmt", [qesgd.FP4_MX, qesgd.FP4_NV])
def test_rows_of_nearly_2_to_31_elements(fmt):
    """One value that the format holds exactly (1; by NV's scales 448 * 2^-11 6 times that) at some places of the longest row there
    may be: its exponent, its values, and its product with itself, a multiple of 2^-8 below 2^16 like all partial sums."""
    cols = qesgd.MAX_MATRIX_SIDE
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("too little memory")
    ctx = G.ctx()
    g = torch.Generator(device="cuda").manual_seed(1)
    at = torch.cat([torch.randint(0, cols, (20_000,), generator=g, device="cuda"), torch.tensor([0, cols - 1, cols - 257, 1 << 30], device="cuda")])
    x = torch.zeros((1, cols), dtype=torch.bfloat16, device="cuda")
    value = 1.0 if fmt == qesgd.FP4_MX else 6 * 448 / 2048
    x[0, at] = value
    e = None
    if fmt == qesgd.FP4_NV:
        e = torch.zeros(1, dtype=torch.int32, device="cuda")
        ctx.qesgd_fp4_tensor_exponent(x, qesgd.BF16, 1, cols, cols, e)
        assert int(e) == ref.tensor_exponent(np.full((1, 1), value)) == -11
    held = qesgd.alloc_fp4(1, cols, fmt, "cuda")
    ctx.qesgd_fp4_quantize(x, qesgd.BF16, 1, cols, cols, fmt, e, 0, 0, 0, 0, *held)
    back = torch.full((1, cols), 5.0, dtype=torch.bfloat16, device="cuda")
    ctx.qesgd_fp4_dequantize(*held, 1, cols, fmt, e, back, qesgd.BF16, cols)
    assert torch.equal(back, x)
    c = torch.empty((1, 1), device="cuda")
    ctx.qesgd_fp4_matmul(*held, e, *held, e, 1, 1, cols, fmt, c, qesgd.F32, 1)
    assert float(c) == value * value * torch.unique(at).numel()
    assert ctx.qesgd_status() == 0
