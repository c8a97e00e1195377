"""The 4-bit quantiser and the tensor's exponent at the ends of every input type: infinities, NaN of either sign, largest and subnormal
numbers, in even and odd columns and rows, and exponents too small for the values."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from oracle import matrix_ref as ref                        # noqa: E402
from paper_1901_03040_b200 import qesgd                     # noqa: E402
from tests import gpu_helpers as G                          # noqa: E402
from tests.test_gpu_matrix_accuracy import WIDE_TOLERANCE  # noqa: E402

DTYPE = {qesgd.F32: torch.float32, qesgd.BF16: torch.bfloat16, qesgd.F16: torch.float16}
FORMATS = [qesgd.FP4_MX, qesgd.FP4_NV]


def _matrix(rows, cols, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((rows, cols), generator=g) * scale).to(DTYPE[dtype])


def _check(x, cols, dtype, fmt, sides, seed, exponent=None, t=0):
    """Codes and scales of the wanted sides against the definition; returns the status word."""
    rows = x.shape[0]
    v = x[:, :cols].double().numpy()
    dev = x.cuda()
    held = {}
    for side, r, c in (("r", rows, cols), ("c", cols, rows)):
        if side in sides:
            held[side] = qesgd.alloc_fp4(r, c, fmt, "cuda")
            for b in held[side]:
                b.fill_(0xAB)
    ctx = G.ctx()
    ctx.qesgd_fp4_quantize(dev, dtype, rows, cols, x.stride(0), fmt, exponent, 0 if seed is None else 1, seed or 0, 2, 3,
                           *held.get("r", (None, None)), *held.get("c", (None, None)))
    for side, (codes, scales) in held.items():
        want_codes, want_bytes, _ = ref.quantize(v if side == "r" else v.T, fmt, t, seed, 2, 3)
        assert (scales.cpu().numpy() == ref.tiles(want_bytes)).all(), side
        assert (codes.cpu().numpy() == ref.pack(want_codes)).all(), side
    return ctx.qesgd_status()


@pytest.mark.parametrize("dtype", list(DTYPE))
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("sides", ["r", "c", "rc"])
def test_non_finite_elements_of_every_type(sides, fmt, dtype):
    """One to a matrix and several, so that a missed one and one that marks a neighbouring block both show."""
    bits = {qesgd.F32: (torch.int32, 0x7F800000, 0x7F800001, 0x7FFFFFFF, -1), qesgd.BF16: (torch.int16, 0x7F80, 0x7F81, 0x7FFF, -1),
            qesgd.F16: (torch.int16, 0x7C00, 0x7C01, 0x7FFF, -1)}[dtype]
    kinds = [float("inf"), float("-inf")] + [torch.tensor([b], dtype=bits[0]).view(DTYPE[dtype]) for b in bits[2:]]
    for n, (rows, cols, pad) in enumerate(((70, 200, 0), (33, 49, 3), (130, 257, 1))):
        for i, kind in enumerate(kinds):
            x = _matrix(rows, cols + pad, dtype, 10 * n + i)
            x[(7 * i + 4) % rows, (16 * i + 8 + i) % cols] = kind                 # even and odd columns, octets' first halves and second
            assert _check(x, cols, dtype, fmt, sides, None if i % 2 else 11) == qesgd.STATUS_NONFINITE
        x = _matrix(rows, cols + pad, dtype, n)
        for i, (r, c) in enumerate(((0, 0), (rows - 1, cols - 1), (3, 40), (20, 41), (rows - 2, 15), (5, 16), (31, 33), (32, 31))):
            x[r, c] = kinds[i % len(kinds)]
        assert _check(x, cols, dtype, fmt, sides, None) == qesgd.STATUS_NONFINITE
        x = _matrix(rows, cols + pad, dtype, n)
        x[:, cols:] = float("nan")                                               # outside the matrix
        assert _check(x, cols, dtype, fmt, sides, 5) == 0


@pytest.mark.parametrize("dtype", list(DTYPE))
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("sides", ["r", "rc"])
def test_largest_and_smallest_numbers_of_every_type(sides, fmt, dtype):
    info = torch.finfo(DTYPE[dtype])
    ends = torch.tensor([info.max, info.min, info.tiny, -info.tiny, info.smallest_normal / 2, -info.smallest_normal * info.eps, 0.0, -0.0, 1.0, -1.0],
                        dtype=torch.float64).to(DTYPE[dtype])
    g = torch.Generator().manual_seed(1)
    for rows, cols, pad in ((64, 96, 0), (50, 131, 1)):
        x = ends[torch.randint(0, len(ends), (rows, cols + pad), generator=g)]
        small = ends[torch.randint(2, 8, (rows, cols + pad), generator=g)]
        x[: rows // 2] = small[: rows // 2]                                       # blocks without anything large
        for seed in (None, 3):
            assert _check(x, cols, dtype, fmt, sides, seed) == 0
    if fmt == qesgd.FP4_NV:
        for given, used in ((-1000, -126), (126, 126), (2 ** 31 - 1, 126), (-126, -126), (20, 20)):
            e = torch.tensor([given], dtype=torch.int32, device="cuda")
            for seed in (None, 3):
                assert _check(x, cols, dtype, fmt, sides, seed, e, used) == 0


@pytest.mark.parametrize("dtype", list(DTYPE))
@pytest.mark.parametrize("sides", ["r", "c", "rc"])
def test_an_exponent_too_small_clips_drawn_values_too(sides, dtype):
    """Scales stop at 448: what is more than 2688 * 2^t ends at 6 times it, whatever the draw; the rest is drawn as ever."""
    x = _matrix(40, 150, dtype, 8)
    x[:, ::5] *= 0.01
    for t in (-12, -8, -10, -126):
        e = torch.tensor([t], dtype=torch.int32, device="cuda")
        for seed in (None, 7):
            assert _check(x, 149, dtype, qesgd.FP4_NV, sides, seed, e, t) == 0


@pytest.mark.parametrize("dtype", list(DTYPE))
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (2, 8, 0), (37, 201, 3), (130, 4100, 1), (300, 2049, 0)])
def test_the_exponent_leaves_non_finite_elements_out(dtype, rows, cols, pad):
    ctx = G.ctx()
    for n, where in enumerate((((0, 0),), ((rows - 1, cols - 1), (0, cols // 2)), ((rows // 2, min(cols - 1, 7)), (rows // 2, min(cols - 1, 8))))):
        x = _matrix(rows, cols + pad, dtype, n, 3.0)
        for i, (r, c) in enumerate(where):
            x[r, c] = (float("inf"), float("nan"), float("-inf"))[(n + i) % 3]
        x[:, cols:] = float("nan")
        dev, e = x.cuda(), torch.full((3,), 77, dtype=torch.int32, device="cuda")
        ctx.qesgd_fp4_tensor_exponent(dev, dtype, rows, cols, cols + pad, e[1:])
        assert e.tolist() == [77, ref.tensor_exponent(x[:, :cols].double().numpy()), 77]
        assert ctx.qesgd_status() == qesgd.STATUS_NONFINITE
    x = _matrix(rows, cols + pad, dtype, 5, 3.0)
    x[:, cols:] = float("nan")
    x[rows // 2, cols // 3] = torch.finfo(DTYPE[dtype]).max
    ctx.qesgd_fp4_tensor_exponent(x.cuda(), dtype, rows, cols, cols + pad, e[1:])
    assert int(e[1]) == ref.tensor_exponent(x[:, :cols].double().numpy()) and ctx.qesgd_status() == 0


@pytest.mark.parametrize("dtype", list(DTYPE))
@pytest.mark.parametrize("rows,cols", [(40, 72), (100, 1000), (150, 300), (300, 150), (600, 530)])
def test_orthogonalize_of_zeros_non_finite_and_far_scales(rows, cols, dtype):
    """In the one-kernel form, alone and by clusters, and as products of their own: a matrix of a batch that is not finite, or
    zero, gives zeros and leaves the others alone; elements near the type's ends are divided by their norm as any; what lies behind a
    row's end is not looked at."""
    pad, batch = 3, 7
    info = torch.finfo(DTYPE[dtype])
    x = _matrix(batch * rows, cols + pad, dtype, 3).view(batch, rows, cols + pad)
    x[0] = 0.0
    x[1, rows - 1, cols - 1] = float("nan")
    x[2, 0, cols // 2] = float("-inf")
    x[3] = (x[3].double().clamp(-1, 1) * info.max).to(DTYPE[dtype])
    x[4] = (x[4].double() * info.tiny * 4).to(DTYPE[dtype])                 # subnormal for the most part
    x[5] = 0.0
    x[5, rows // 2, cols // 3] = info.smallest_normal * info.eps            # the smallest number there is
    x[:, :, cols:] = float("nan")
    dev = x.cuda()
    out = torch.full((batch, rows, cols + 1), 9.0, dtype=torch.bfloat16, device="cuda")
    need = qesgd.orthogonalize_workspace(rows, cols, batch)
    work = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    ctx = G.ctx()
    ctx.qesgd_orthogonalize(dev, dtype, rows, cols, cols + pad, batch, x.stride(0), 5, out, cols + 1, rows * (cols + 1), work, need)
    assert ctx.qesgd_status() == qesgd.STATUS_NONFINITE
    assert (out[:, :, cols:] == 9.0).all() and (out[:3, :, :cols] == 0).all()
    for i in (3, 4, 5, 6):
        want = ref.orthogonalize(x[i, :, :cols].double().numpy())
        off = np.linalg.norm(out[i, :, :cols].double().cpu().numpy() - want) / np.linalg.norm(want)
        assert off <= WIDE_TOLERANCE, (i, off)
    x[1:3] = 0.0
    ctx.qesgd_orthogonalize(x.cuda(), dtype, rows, cols, cols + pad, batch, x.stride(0), 5, out, cols + 1, rows * (cols + 1), work, need)
    assert ctx.qesgd_status() == 0
