"""The matrix operators on the GPU against a plain implementation in 64 bits: microscaled 4-bit floats bit for bit, their
product, the orthogonalised update, and a whole training round of a weight matrix built of them."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from oracle import matrix_ref as ref                        # noqa: E402
from paper_1901_03040_b200 import qesgd                     # noqa: E402
from tests import gpu_helpers as G                          # noqa: E402

DTYPE = {qesgd.F32: torch.float32, qesgd.BF16: torch.bfloat16, qesgd.F16: torch.float16}
FORMATS = [qesgd.FP4_MX, qesgd.FP4_NV]
SIZES = [(1, 1), (1, 16), (3, 33), (128, 64), (129, 130), (1, 4096), (300, 257), (64, 1000), (257, 31)]


def _x(rows, cols, dtype, seed, pad=0, scale=1e-3):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols + pad), generator=g) * scale
    x[torch.rand((rows, cols + pad), generator=g) < 0.02] *= 30.0
    x[torch.rand((rows, cols + pad), generator=g) < 0.05] = 0.0
    return x.to(DTYPE[dtype]).cuda()


def _np(t):
    return t.detach().cpu().double().numpy()


def _quantize(x, cols, fmt, sides, seed=None, worker=0, epoch=0, exponent=None, dtype=None):
    """Codes and scales of the wanted sides ("r", "c"), with canaries around every output; and the status word."""
    rows = x.shape[0]
    held, bufs = {}, []
    for side, r, c in (("r", rows, cols), ("c", cols, rows)):
        if side in sides:
            rb, sb = qesgd.fp4_row_bytes(c), qesgd.fp4_scale_bytes(r, c, fmt)
            codes = torch.full((16 + r * rb + 16,), 0xAB, dtype=torch.uint8, device="cuda")
            scales = torch.full((16 + sb + 16,), 0xAB, dtype=torch.uint8, device="cuda")
            held[side] = (codes[16:16 + r * rb].view(r, rb), scales[16:16 + sb])
            bufs += [codes, scales]
    ctx = G.ctx()
    ctx.qesgd_fp4_quantize(x, dtype, rows, cols, x.stride(0), fmt, exponent,
                           qesgd.ROUND_NEAREST if seed is None else qesgd.ROUND_STOCHASTIC, seed or 0, worker, epoch,
                           *held.get("r", (None, None)), *held.get("c", (None, None)))
    status = ctx.qesgd_status()
    for b in bufs:
        assert (b[:16] == 0xAB).all() and (b[-16:] == 0xAB).all(), "wrote outside its buffer"
    return held, status


def _check_held(held, x, fmt, t=0, seed=None, worker=0, epoch=0):
    for side, (codes, scales) in held.items():
        want_codes, want_bytes, _ = ref.quantize(x if side == "r" else x.T, fmt, t, seed, worker, epoch)
        got = scales.cpu().numpy()
        bad = np.nonzero(got != ref.tiles(want_bytes))[0]
        assert bad.size == 0, f"{side}: {bad.size} scale bytes differ, first {bad[:4]}: {got[bad[:4]]}"
        bad = np.argwhere(codes.cpu().numpy() != ref.pack(want_codes))
        assert bad.size == 0, f"{side}: {len(bad)} code bytes differ, first {bad[:4].tolist()}"


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", list(DTYPE))
@pytest.mark.parametrize("fmt", FORMATS)
def test_quantize_nearest(fmt, dtype, rows, cols):
    for pad, sides in ((0, "rc"), (1, "r"), (8, "c"), (3, "rc")):
        x = _x(rows, cols, dtype, rows + cols + pad, pad)
        held, status = _quantize(x, cols, fmt, sides, dtype=dtype)
        assert status == 0
        _check_held(held, _np(x)[:, :cols], fmt)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", list(DTYPE))
@pytest.mark.parametrize("fmt", FORMATS)
def test_quantize_stochastic(fmt, dtype, rows, cols):
    for pad, sides, seed in ((0, "rc", 7), (1, "r", 0x123456789ABCDEF0), (8, "c", (1 << 64) - 1)):
        x = _x(rows, cols, dtype, rows * cols + pad, pad)
        held, status = _quantize(x, cols, fmt, sides, seed, 3, 0xFFFFFFFF, dtype=dtype)
        assert status == 0
        _check_held(held, _np(x)[:, :cols], fmt, 0, seed, 3, 0xFFFFFFFF)


@pytest.mark.parametrize("seed", [None, 11])
@pytest.mark.parametrize("rows,cols,dtype", [(129, 40001, qesgd.BF16), (1000, 4800, qesgd.F32)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_quantize_of_many_tiles(fmt, rows, cols, dtype, seed):
    """More tiles of 64 rows than run at once: smaller matrices take tiles of 32."""
    x = _x(rows, cols, dtype, 21, 3)
    held, status = _quantize(x, cols, fmt, "r", seed, 1, 2, dtype=dtype)
    assert status == 0
    _check_held(held, _np(x)[:, :cols], fmt, 0, seed, 1, 2)


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_border_of_the_grid_and_of_the_scales(fmt):
    """Blocks whose largest magnitude runs over all scale borders (6 times a scale and its neighbours in fp32), with
    elements on and next to every border between two codes."""
    scales = ref.E8M0[::7] if fmt == qesgd.FP4_MX else ref.E4M3[1:]
    size = ref.BLOCK[fmt]
    rows = []
    for s in scales:
        for top in (6.0 * s, np.nextafter(np.float32(6.0 * s), np.float32(np.inf)), np.nextafter(np.float32(6.0 * s), np.float32(0))):
            if not np.isfinite(np.float32(top)):
                continue
            edges = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]) * s
            e32 = edges.astype(np.float32)
            near = np.concatenate([[np.float32(top)], e32, -np.nextafter(e32, np.float32(np.inf)), np.nextafter(e32, np.float32(0))])
            rows += [near[:1].tolist() + near[k:k + size - 1].tolist() for k in (1, 8)]
    x = np.zeros((len(rows), size), dtype=np.float32)
    for i, r in enumerate(rows):
        x[i, :len(r)] = r[:size]
    t = torch.from_numpy(x).cuda()
    for seed in (None, 5):
        held, status = _quantize(t, size, fmt, "rc", seed, dtype=qesgd.F32)
        assert status == 0
        _check_held(held, x.astype(np.float64), fmt, 0, seed)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kind", ["zeros", "subnormal", "huge", "tiny", "nonfinite"])
def test_quantize_extremes(fmt, kind):
    x = _np(_x(70, 200, qesgd.F32, 4)).astype(np.float32)
    if kind == "zeros":
        x[:, 32:96] = 0.0
        x[5] = -0.0
    if kind == "subnormal":
        x = (x * 1e-38).astype(np.float32)
        x[0, :8] = [1e-45, -1e-45, 1.2e-38, 0, 5e-39, -2e-40, 1e-44, 3e-45]
    if kind == "huge":
        x = np.clip(x.astype(np.float64) * 1e40, -3.4e38, 3.4e38).astype(np.float32)
    if kind == "tiny":
        x = (x * 1e-20).astype(np.float32)
    if kind == "nonfinite":
        x[3, 40], x[9, 0], x[69, 199], x[20, 64] = np.inf, np.nan, -np.inf, np.nan
    for seed in (None, 11):
        held, status = _quantize(torch.from_numpy(x).cuda(), 200, fmt, "rc", seed, dtype=qesgd.F32)
        assert status == (qesgd.STATUS_NONFINITE if kind == "nonfinite" else 0)
        _check_held(held, x.astype(np.float64), fmt, 0, seed)


@pytest.mark.parametrize("dtype", list(DTYPE))
@pytest.mark.parametrize("rows,cols,pad,scale", [(1, 1, 0, 1e-6), (37, 201, 3, 1e-4), (300, 1000, 0, 100.0), (2, 8, 0, 0.0)])
def test_tensor_exponent_and_quantize_by_it(dtype, rows, cols, pad, scale):
    x = _x(rows, cols, dtype, 3, pad, scale)
    x[:, cols:] = 1e4                                    # outside the matrix
    e = torch.full((3,), 77, dtype=torch.int32, device="cuda")
    G.ctx().qesgd_fp4_tensor_exponent(x, dtype, rows, cols, x.stride(0), e[1:])
    v = _np(x)[:, :cols]
    want = ref.tensor_exponent(v)
    assert e.tolist() == [77, want, 77]
    for seed in (None, 2):
        held, status = _quantize(x, cols, qesgd.FP4_NV, "rc", seed, exponent=e[1:], dtype=dtype)
        assert status == 0
        _check_held(held, v, qesgd.FP4_NV, want, seed)


def test_tensor_exponent_borders_and_nonfinite():
    ctx = G.ctx()
    e = torch.zeros(1, dtype=torch.int32, device="cuda")
    for t in (-130, -126, -125, -30, 0, 40, 116):
        for f in (2688.0, float(np.nextafter(np.float32(2688), np.float32(1e9)))):
            x = torch.tensor([[0.0, -f * 2.0 ** t]], dtype=torch.float64).float().cuda()
            ctx.qesgd_fp4_tensor_exponent(x, qesgd.F32, 1, 2, 2, e)
            assert int(e) == ref.tensor_exponent(_np(x)), (t, f)
    assert ctx.qesgd_status() == 0
    x = torch.tensor([[1.0, float("inf")], [float("nan"), 5000.0]], device="cuda")
    ctx.qesgd_fp4_tensor_exponent(x, qesgd.F32, 2, 2, 2, e)
    assert int(e) == 1 and ctx.qesgd_status() == qesgd.STATUS_NONFINITE


def test_an_exponent_outside_its_range_is_clamped_and_one_too_small_clips():
    x = _x(40, 64, qesgd.F32, 1, 0, 1.0)
    for given, used in ((-1000, -126), (2 ** 31 - 1, 126), (-8, -8)):
        e = torch.tensor([given], dtype=torch.int32, device="cuda")
        held, status = _quantize(x, 64, qesgd.FP4_NV, "rc", None, exponent=e, dtype=qesgd.F32)
        assert status == 0
        _check_held(held, _np(x), qesgd.FP4_NV, used)


def test_stochastic_rounding_is_unbiased():
    """The mean over N epochs of a value on a grid of spacing h lies within 6 standard errors, 6 h / (2 sqrt(N)), of
    it for each of the 4096 elements (6 sigma: 2e-9 each, 2e-5 over all of them and both formats)."""
    x = _x(8, 512, qesgd.F32, 9)
    N = 400
    for fmt in FORMATS:
        total = np.zeros((8, 512))
        for epoch in range(N):
            held, _ = _quantize(x, 512, fmt, "r", 77, 0, epoch, dtype=qesgd.F32)
            out = torch.empty((8, 512), device="cuda")
            G.ctx().qesgd_fp4_dequantize(*held["r"], 8, 512, fmt, None, out, qesgd.F32, 512)
            total += _np(out)
        _, byte, _ = ref.quantize(_np(x), fmt)
        scale = np.repeat((ref.E8M0 if fmt == qesgd.FP4_MX else ref.E4M3)[byte], ref.BLOCK[fmt], 1)
        q = np.abs(_np(x)) / scale
        h = np.where(q < 2, 0.5, np.where(q < 4, 1.0, 2.0)) * scale
        assert (np.abs(total / N - _np(x)) <= 6 * h / (2 * np.sqrt(N)) + 1e-12).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_dequantize_of_all_codes_and_scales(fmt, rows, cols):
    g = np.random.default_rng(rows * 1000 + cols)
    codes = g.integers(0, 16, (rows, cols), dtype=np.uint8)
    byte = g.integers(0, 254 if fmt == qesgd.FP4_MX else 127, (rows, -(-cols // ref.BLOCK[fmt])), dtype=np.uint8)
    t = 0 if fmt == qesgd.FP4_MX else -3
    e = None if fmt == qesgd.FP4_MX else torch.tensor([t], dtype=torch.int32, device="cuda")
    want = torch.from_numpy(ref.values(codes, byte, fmt, t))
    dc, ds = G.dev(ref.pack(codes)), G.dev(ref.tiles(byte))
    for dtype in DTYPE:
        for ld in (cols, cols + 1, cols + 8):
            out = torch.full((rows, ld), 55.0, dtype=DTYPE[dtype], device="cuda")
            G.ctx().qesgd_fp4_dequantize(dc, ds, rows, cols, fmt, e, out, dtype, ld)
            torch.cuda.synchronize()
            assert torch.equal(out[:, :cols].cpu(), want.to(DTYPE[dtype]))
            assert (out[:, cols:] == 55.0).all()


# ---------------------------------------------------------------- product ----
def _operand(rows, K, fmt, seed, exact):
    """Random codes; scales such that every product and sum is a multiple of 2^-4 below 2^20 (exact), or any."""
    g = np.random.default_rng(seed)
    codes = g.integers(0, 16, (rows, K), dtype=np.uint8)
    nb = -(-K // ref.BLOCK[fmt])
    if exact:
        # 1/2, 1, 2; for E4M3 1/2, 1, 1.5
        pick = np.array([126, 127, 128] if fmt == qesgd.FP4_MX else [0x30, 0x38, 0x3C], dtype=np.uint8)
        byte = pick[g.integers(0, 3, (rows, nb))]
    else:
        byte = g.integers(*((117, 130) if fmt == qesgd.FP4_MX else (0, 127)), (rows, nb), dtype=np.uint8)
    return ref.values(codes, byte, fmt), G.dev(ref.pack(codes)), G.dev(ref.tiles(byte))


PRODUCTS = [(1, 1, 1), (1, 16, 32), (1, 128, 64), (1, 300, 4096), (5, 1000, 513), (17, 129, 100), (64, 256, 2048), (128, 128, 256),
            (129, 257, 65), (200, 40, 1000), (256, 256, 512), (300, 520, 700), (513, 1030, 321), (1000, 64, 33)]


@pytest.mark.parametrize("M,N,K", PRODUCTS)
@pytest.mark.parametrize("fmt", FORMATS)
def test_product_of_exact_sums(fmt, M, N, K):
    """Every partial sum in any order is exact in fp32 (multiples of 2^-4 below 12 * 12 * 4096 < 2^20): the result is
    the exact one rounded once to the output's type.  Rows of C wider than N keep what lies behind them."""
    a, ca, sa = _operand(M, K, fmt, M + K, True)
    b, cb, sb = _operand(N, K, fmt, N + 7 * K, True)
    want = torch.from_numpy(a @ b.T)
    for dtype, pad, acc in ((qesgd.F32, 0, 0), (qesgd.F32, 3, 1), (qesgd.BF16, 1, 0), (qesgd.BF16, 8, 1), (qesgd.F16, 0, 1), (qesgd.F16, 5, 0)):
        c = torch.randint(-8, 9, (M, N + pad), generator=torch.Generator().manual_seed(N)).to(DTYPE[dtype]).cuda()
        before = c.clone()
        G.ctx().qesgd_fp4_matmul(ca, sa, None, cb, sb, None, M, N, K, fmt, c, dtype, N + pad, acc)
        torch.cuda.synchronize()
        full = want + (before[:, :N].cpu().double() if acc else 0.0)
        assert torch.equal(c[:, :N].cpu(), full.to(DTYPE[dtype])), (dtype, pad, acc)
        assert torch.equal(c[:, N:], before[:, N:])
    assert G.ctx().qesgd_status() == 0


@pytest.mark.parametrize("M,N,K", [(2100, 2400, 300), (2304, 2500, 3000), (9000, 520, 65)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_product_of_many_tiles(fmt, M, N, K):
    """Enough tiles that pairs of SMs share them: exact sums, as above."""
    a, ca, sa = _operand(M, K, fmt, 5, True)
    b, cb, sb = _operand(N, K, fmt, 6, True)
    want = torch.from_numpy(a @ b.T)
    for dtype, pad, acc in ((qesgd.F32, 1, 1), (qesgd.BF16, 0, 0)):
        c = torch.randint(-8, 9, (M, N + pad), generator=torch.Generator().manual_seed(N)).to(DTYPE[dtype]).cuda()
        before = c.clone()
        G.ctx().qesgd_fp4_matmul(ca, sa, None, cb, sb, None, M, N, K, fmt, c, dtype, N + pad, acc)
        torch.cuda.synchronize()
        full = want + (before[:, :N].cpu().double() if acc else 0.0)
        assert torch.equal(c[:, :N].cpu(), full.to(DTYPE[dtype])), (dtype, pad, acc)
        assert torch.equal(c[:, N:], before[:, N:])
    assert G.ctx().qesgd_status() == 0


@pytest.mark.parametrize("M,N,K", [(1, 2500, 20000), (64, 1000, 65536), (40, 130, 40000), (150, 700, 30001)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_product_of_a_long_contraction(fmt, M, N, K):
    """Values up to 1.5 and scales of one: sums are multiples of 1/4 below 2.25 * 65536 < 2^18, exact in any order."""
    g = np.random.default_rng(K)
    held = []
    for rows in (M, N):
        codes = g.integers(0, 4, (rows, K), dtype=np.uint8) + 8 * g.integers(0, 2, (rows, K), dtype=np.uint8)
        byte = np.full((rows, -(-K // ref.BLOCK[fmt])), 127 if fmt == qesgd.FP4_MX else 0x38, dtype=np.uint8)
        held.append((ref.values(codes, byte, fmt), G.dev(ref.pack(codes)), G.dev(ref.tiles(byte))))
    (a, ca, sa), (b, cb, sb) = held
    c = torch.empty((M, N), device="cuda")
    G.ctx().qesgd_fp4_matmul(ca, sa, None, cb, sb, None, M, N, K, fmt, c, qesgd.F32, N, 0)
    assert torch.equal(c.cpu().double(), torch.from_numpy(a @ b.T))
    assert G.ctx().qesgd_status() == 0


@pytest.mark.parametrize("M,N,K", [(1, 200, 3000), (33, 333, 1111), (300, 400, 2000)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_product_of_any_scales(fmt, M, N, K):
    """K additions in fp32, each off by at most one unit (2^-23, rounded or cut) of a partial sum that sum |a||b| bounds."""
    a, ca, sa = _operand(M, K, fmt, 1, False)
    b, cb, sb = _operand(N, K, fmt, 2, False)
    e = None if fmt == qesgd.FP4_MX else torch.tensor([3, -7], dtype=torch.int32, device="cuda")
    power = 1.0 if e is None else 2.0 ** -4
    c = torch.empty((M, N), device="cuda")
    G.ctx().qesgd_fp4_matmul(ca, sa, e if e is None else e[:1], cb, sb, e if e is None else e[1:], M, N, K, fmt, c, qesgd.F32, N, 0)
    off = np.abs(_np(c) - power * (a @ b.T))
    assert (off <= (K + 4) * 2.0 ** -23 * power * (np.abs(a) @ np.abs(b).T)).all()
    # all but a few of the additions lose nothing near that: the errors of a sum of independent roundings
    assert np.sqrt(np.mean(off ** 2)) <= 4 * np.sqrt(K) * 2.0 ** -23 * power * np.sqrt(np.mean((np.abs(a) @ np.abs(b).T) ** 2))


def test_product_over_nothing():
    c = torch.full((3, 5), 2.0, device="cuda")
    ctx = G.ctx()
    ctx.qesgd_fp4_matmul(None, None, None, None, None, None, 3, 4, 0, qesgd.FP4_MX, c, qesgd.F32, 5, 1)
    torch.cuda.synchronize()
    assert (c == 2.0).all()
    ctx.qesgd_fp4_matmul(None, None, None, None, None, None, 3, 4, 0, qesgd.FP4_MX, c, qesgd.F32, 5, 0)
    torch.cuda.synchronize()
    assert (c[:, :4] == 0.0).all() and (c[:, 4] == 2.0).all()


# -------------------------------------------------------------- orthogonal ----
# What five steps may be off, as a share of the result's 2-norm: the result's rounding to bf16, at most 2^-8, and in
# each step two roundings of fp16 operands (X, and what is off the diagonal of B), at most 2^-11 of the term they
# enter; the steps that follow enlarge signal and error alike.
ORTHO_TOLERANCE = 2.0 ** -8 + 5 * 2 * 2.0 ** -11


def _orthogonalize(x, dtype, rows, cols, batch=1, steps=5, ldo=None, ctx=None, **coefficients):
    need = qesgd.orthogonalize_workspace(rows, cols, batch)
    work = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")     # NaN in every type
    ldo = ldo or cols
    out = torch.full((batch, rows, ldo), 9.0, dtype=torch.bfloat16, device="cuda")
    (ctx or G.ctx()).qesgd_orthogonalize(x, dtype, rows, cols, x.stride(-2), batch, x.stride(0) if batch > 1 else 0, steps, out,
                                         ldo, rows * ldo, work, need, **coefficients)
    torch.cuda.synchronize()
    assert (work[need:] == 0xFF).all() and (out[:, :, cols:] == 9.0).all()
    return out[:, :, :cols]


def _gradient(batch, rows, cols, dtype, seed, pad=0):
    g = torch.Generator().manual_seed(seed)
    k = min(8, rows, cols)
    x = torch.randn((batch, rows, cols + pad), generator=g)
    x = x + 0.5 * torch.randn((batch, rows, k), generator=g) @ torch.randn((batch, k, cols + pad), generator=g)
    return (x * 1e-4 if dtype != qesgd.F16 else x).to(DTYPE[dtype]).cuda()


@pytest.mark.parametrize("rows,cols", [(16, 16), (17, 31), (64, 256), (256, 64), (100, 1000), (128, 128), (129, 300), (300, 129),
                                       (256, 512), (500, 500), (520, 1030), (1000, 130), (128, 4096), (2100, 90), (70, 520), (40, 4500), (4500, 40)])
@pytest.mark.parametrize("dtype", list(DTYPE))
def test_orthogonalize(dtype, rows, cols):
    for batch, pad, ldo in ((1, 0, None), (3, 1, cols + 3), (2, 8, cols + 8)):
        x = _gradient(batch, rows, cols, dtype, rows + cols, pad)
        got = _np(_orthogonalize(x, dtype, rows, cols, batch, ldo=ldo))
        for i in range(batch):
            want = ref.orthogonalize(_np(x[i, :, :cols]))
            assert np.linalg.norm(got[i] - want) <= ORTHO_TOLERANCE * np.linalg.norm(want)
    assert G.ctx().qesgd_status() == 0


@pytest.mark.parametrize("rows,cols,batch", [(100, 3000, 16), (100, 3000, 5), (2000, 64, 40), (128, 128, 200), (120, 700, 50)])
def test_orthogonalize_of_many_small_matrices(rows, cols, batch):
    """More clusters than the device runs at once, and the batch sizes around which single products take over."""
    x = _gradient(batch, rows, cols, qesgd.BF16, 4)
    got = _np(_orthogonalize(x, qesgd.BF16, rows, cols, batch))
    for i in range(0, batch, 1 + batch // 10):
        want = ref.orthogonalize(_np(x[i]))
        assert np.linalg.norm(got[i] - want) <= ORTHO_TOLERANCE * np.linalg.norm(want)


@pytest.mark.parametrize("rows,cols", [(600, 900), (900, 600), (513, 513)])
def test_orthogonalize_of_many_larger_matrices(rows, cols):
    """Enough tiles that pairs of SMs share them, in all three products."""
    x = _gradient(14, rows, cols, qesgd.BF16, 2, 3)
    got = _np(_orthogonalize(x, qesgd.BF16, rows, cols, 14))
    for i in range(14):
        want = ref.orthogonalize(_np(x[i, :, :cols]))
        assert np.linalg.norm(got[i] - want) <= ORTHO_TOLERANCE * np.linalg.norm(want)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 50), (50, 1), (2, 3), (5, 700), (15, 15)])
def test_orthogonalize_of_few_rows(rows, cols):
    x = _gradient(2, rows, cols, qesgd.F32, 5)
    got = _np(_orthogonalize(x, qesgd.F32, rows, cols, 2))
    for i in range(2):
        want = ref.orthogonalize(_np(x[i]))
        assert np.linalg.norm(got[i] - want) <= ORTHO_TOLERANCE * np.linalg.norm(want)


@pytest.mark.parametrize("rows,cols", [(48, 500), (500, 40), (32, 4000), (33, 257), (3000, 20), (64, 64), (16, 200), (10, 256), (65, 190)])
def test_orthogonalize_where_quarters_share_rows(rows, cols):
    """Up to 32 and up to 64 rows of the smaller side, for which the update of a row is taken out by several warps."""
    x = _gradient(3, rows, cols, qesgd.F32, 6, 2)
    for steps in (1, 2, 5):
        got = _np(_orthogonalize(x, qesgd.F32, rows, cols, 3, steps))
        for i in range(3):
            want = ref.orthogonalize(_np(x[i, :, :cols]), steps)
            assert np.linalg.norm(got[i] - want) <= ORTHO_TOLERANCE * np.linalg.norm(want)


def test_orthogonalize_steps_and_coefficients():
    x = _gradient(1, 150, 260, qesgd.F32, 1)
    for steps, abc in ((1, (3.4445, -4.7750, 2.0315)), (2, (1.5, -0.5, 0.0)), (12, (1.5, -0.5, 0.0)), (3, (2.0, -1.5, 0.5)),
                       (32, (1.875, -1.25, 0.375))):
        got = _np(_orthogonalize(x, qesgd.F32, 150, 260, 1, steps, a=abc[0], b=abc[1], c=abc[2]))[0]
        want = ref.orthogonalize(_np(x[0]), steps, *abc)
        assert np.linalg.norm(got - want) <= (2.0 ** -8 + steps * 2 * 2.0 ** -11) * np.linalg.norm(want)


@pytest.mark.parametrize("rows,cols", [(8, 16), (60, 250), (128, 700), (200, 300)])
def test_orthogonalize_of_growing_singular_values_stays_finite(rows, cols):
    """Coefficients that multiply by 16 a step: what is kept between steps is cut off at 65504 / 256, so that the last step's
    terms are at most |a + b d + c (A A + d d)| 256 with d below cols 256^2, far inside bf16's range."""
    x = _gradient(2, rows, cols, qesgd.F32, 9)
    for a, b, c in ((16.0, 0.0, 0.0), (16.0, 32.0, 32.0), (-16.0, -32.0, -32.0)):
        got = _orthogonalize(x, qesgd.F32, rows, cols, 2, 16, a=a, b=b, c=c)
        assert torch.isfinite(got).all() and (got != 0).any()
    assert G.ctx().qesgd_status() == 0


def test_orthogonalize_with_far_singular_values():
    """Sixteen directions 160 times as strong as the rest: the rest has to come out right too."""
    g = torch.Generator().manual_seed(0)
    x = 0.1 * torch.randn((512, 512), generator=g) + torch.randn((512, 16), generator=g) @ torch.randn((16, 512), generator=g)
    got = _np(_orthogonalize(x.cuda()[None], qesgd.F32, 512, 512))[0]
    want = ref.orthogonalize(x.double().numpy())
    assert np.linalg.norm(got - want) <= ORTHO_TOLERANCE * np.linalg.norm(want)


def test_orthogonalize_zeros_nonfinite_and_extreme_scales():
    x = _gradient(6, 40, 72, qesgd.F32, 3)
    x[0] = 0.0
    x[1, 3, 5] = float("nan")
    x[2, 39, 71] = float("-inf")
    x[3] *= 1e-36
    x[4] *= 1e38
    before = x.clone()
    got = _orthogonalize(x, qesgd.F32, 40, 72, 6)
    assert G.ctx().qesgd_status() == qesgd.STATUS_NONFINITE
    assert (got[:3] == 0).all() and torch.equal(x.nan_to_num(), before.nan_to_num())
    for i in (3, 4, 5):
        want = ref.orthogonalize(_np(x[i]))
        assert np.linalg.norm(_np(got[i]) - want) <= ORTHO_TOLERANCE * np.linalg.norm(want)


def test_orthogonalize_in_place_twice_and_a_row_of_one():
    x = _gradient(1, 130, 200, qesgd.BF16, 8)
    first = _orthogonalize(x, qesgd.BF16, 130, 200)
    again = _orthogonalize(x, qesgd.BF16, 130, 200)
    assert torch.equal(first, again)
    need = qesgd.orthogonalize_workspace(130, 200)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    y = x[0].clone()
    G.ctx().qesgd_orthogonalize(y, qesgd.BF16, 130, 200, 200, 1, 0, 5, y, 200, 0, work, need)
    torch.cuda.synchronize()
    assert torch.equal(y, first[0])


# ------------------------------------------------- streams, graphs, errors ----
def test_other_streams_and_captured_graphs():
    """Two contexts on two streams at once, each with its own workspace; then each captured and replayed on new inputs."""
    rows, cols = 192, 320
    ctxs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    xs = [_gradient(1, rows, cols, qesgd.F32, 30 + i)[0] for i in range(2)]
    eager = []
    for i in range(2):
        held, _ = _quantize(xs[i], cols, qesgd.FP4_NV, "rc", dtype=qesgd.F32)
        c = torch.empty((rows, rows), device="cuda")
        G.ctx().qesgd_fp4_matmul(*held["r"], None, *held["r"], None, rows, rows, cols, qesgd.FP4_NV, c, qesgd.F32, rows)
        o = _orthogonalize(xs[i][None], qesgd.F32, rows, cols)[0].clone()
        eager.append((held["r"][0].clone(), c.clone(), o))
    state = []
    for i in range(2):
        ctx = qesgd.Context(0, streams[i])
        ctxs.append(ctx)
        need = qesgd.orthogonalize_workspace(rows, cols)
        state.append(dict(x=torch.zeros_like(xs[i]), codes=qesgd.alloc_fp4(rows, cols, qesgd.FP4_NV, "cuda"),
                          e=torch.zeros(1, dtype=torch.int32, device="cuda"), c=torch.empty((rows, rows), device="cuda"),
                          o=torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda"),
                          work=torch.empty(need, dtype=torch.uint8, device="cuda"), need=need))
    torch.cuda.synchronize()

    def run(i):
        s = state[i]
        ctxs[i].qesgd_fp4_quantize(s["x"], qesgd.F32, rows, cols, cols, qesgd.FP4_NV, None, 0, 0, 0, 0, *s["codes"])
        ctxs[i].qesgd_fp4_matmul(*s["codes"], None, *s["codes"], None, rows, rows, cols, qesgd.FP4_NV, s["c"], qesgd.F32, rows)
        ctxs[i].qesgd_fp4_tensor_exponent(s["x"], qesgd.F32, rows, cols, cols, s["e"])
        ctxs[i].qesgd_orthogonalize(s["x"], qesgd.F32, rows, cols, cols, 1, 0, 5, s["o"], cols, 0, s["work"], s["need"])

    def check():
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(state[i]["codes"][0], eager[i][0])
            assert torch.equal(state[i]["c"], eager[i][1]) and torch.equal(state[i]["o"], eager[i][2])
            assert int(state[i]["e"]) == ref.tensor_exponent(_np(xs[i]))

    for i in range(2):
        state[i]["x"].copy_(xs[i])
    torch.cuda.synchronize()
    for _ in range(3):
        for i in range(2):
            run(i)
    check()
    graphs = []
    for i in range(2):
        state[i]["x"].zero_()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[i]):
            run(i)
        graphs.append(g)
    for i in range(2):
        state[i]["x"].copy_(xs[i])
        for v in (state[i]["c"], state[i]["o"]):
            v.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
    check()
    for c in ctxs:
        assert c.qesgd_status() == 0
        c.close()


_FIRST_CALLS = r"""
import sys, torch
sys.path.insert(0, sys.argv[1])
from paper_1901_03040_b200 import qesgd
torch.cuda.set_device(0)
stream = torch.cuda.Stream()
ctx = qesgd.Context(0, stream)
x = torch.randn(130, 300, device="cuda")
codes, scales = qesgd.alloc_fp4(130, 300, qesgd.FP4_NV, "cuda")
codes_t, scales_t = qesgd.alloc_fp4(300, 130, qesgd.FP4_NV, "cuda")
e = torch.zeros(1, dtype=torch.int32, device="cuda")
c, back = torch.zeros(130, 130, device="cuda"), torch.zeros(130, 300, device="cuda")
o, small = torch.zeros(130, 300, dtype=torch.bfloat16, device="cuda"), torch.zeros(20, 300, dtype=torch.bfloat16, device="cuda")
need = qesgd.orthogonalize_workspace(130, 300)
work = torch.empty(need, dtype=torch.uint8, device="cuda")
def run():
    ctx.qesgd_fp4_tensor_exponent(x, 0, 130, 300, 300, e)
    ctx.qesgd_fp4_quantize(x, 0, 130, 300, 300, qesgd.FP4_NV, e, 1, 7, 0, 0, codes, scales, codes_t, scales_t)
    ctx.qesgd_fp4_dequantize(codes, scales, 130, 300, qesgd.FP4_NV, e, back, 0, 300)
    ctx.qesgd_fp4_matmul(codes, scales, e, codes, scales, e, 130, 130, 300, qesgd.FP4_NV, c, 0, 130)
    ctx.qesgd_orthogonalize(x, 0, 130, 300, 300, 1, 0, 5, o, 300, 0, work, need)
    ctx.qesgd_orthogonalize(x, 0, 20, 300, 300, 1, 0, 5, small, 300, 0, work, need)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g, stream=stream):
    run()
g.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (codes, codes_t, back, c, o, small)]
for t in (codes, codes_t, back, c, o, small):
    t.zero_()
torch.cuda.synchronize()
run()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, (codes, codes_t, back, c, o, small)))
assert float(o.float().abs().sum()) > 0 and ctx.qesgd_status() == 0
ctx.close()
print("first calls captured")
"""


def test_the_first_calls_of_a_process_may_be_captured():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", _FIRST_CALLS, root], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "first calls captured" in out.stdout, (out.stdout + out.stderr)[-3000:]


def test_two_host_threads_with_a_context_each():
    import threading
    rows, cols, errors = 260, 410, []
    want = _np(_orthogonalize(_gradient(1, rows, cols, qesgd.F32, 3), qesgd.F32, rows, cols))
    x = _gradient(1, rows, cols, qesgd.F32, 3)

    def work(i):
        try:
            torch.cuda.set_device(0)
            ctx = qesgd.Context(0, torch.cuda.Stream())
            need = qesgd.orthogonalize_workspace(rows, cols)
            out = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
            ws = torch.empty(need, dtype=torch.uint8, device="cuda")
            torch.cuda.synchronize()
            for _ in range(20):
                ctx.qesgd_orthogonalize(x, qesgd.F32, rows, cols, cols, 1, 0, 5, out, cols, 0, ws, need)
            assert ctx.qesgd_status() == 0
            if not (_np(out) == want[0]).all():
                errors.append(i)
            ctx.close()
        except Exception as exc:  # noqa: BLE001
            errors.append(exc)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors


def test_offsets_beyond_32_bits():
    """Rows so far apart that their offsets pass 2^32 elements: quantise, dequantise, product, orthogonal update."""
    rows, cols, ld = 140, 300, 32_000_001            # 4.48e9 elements, 9 GB
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("too little memory")
    buf = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (rows, cols), (ld, 1))
    x.copy_(_x(rows, cols, qesgd.BF16, 5))
    small = x.contiguous()
    ctx = G.ctx()
    for fmt in FORMATS:
        far, _ = _quantize(x, cols, fmt, "rc", dtype=qesgd.BF16)
        _check_held(far, _np(small), fmt)
        near = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
        ctx.qesgd_fp4_dequantize(*far["r"], rows, cols, fmt, None, near, qesgd.BF16, cols)
        product = torch.empty((rows, rows), dtype=torch.bfloat16, device="cuda")
        ctx.qesgd_fp4_matmul(*far["r"], None, *far["r"], None, rows, rows, cols, fmt, product, qesgd.BF16, rows)
        o = _orthogonalize(small[None], qesgd.BF16, rows, cols)[0]
        for view, want, call in (
                ((rows, cols), near, lambda v: ctx.qesgd_fp4_dequantize(*far["r"], rows, cols, fmt, None, v, qesgd.BF16, ld)),
                ((rows, rows), product, lambda v: ctx.qesgd_fp4_matmul(*far["r"], None, *far["r"], None, rows, rows, cols, fmt, v, qesgd.BF16, ld))):
            v = torch.as_strided(buf, view, (ld, 1))
            call(v)
            assert torch.equal(v, want)
        x.copy_(small)
        need = qesgd.orthogonalize_workspace(rows, cols)
        work = torch.empty(need, dtype=torch.uint8, device="cuda")
        ctx.qesgd_orthogonalize(x, qesgd.BF16, rows, cols, ld, 1, 0, 5, x, ld, 0, work, need)
        assert torch.equal(x, o)
        x.copy_(small)
        e = torch.empty(1, dtype=torch.int32, device="cuda")
        ctx.qesgd_fp4_tensor_exponent(x, qesgd.BF16, rows, cols, ld, e)
        assert int(e) == ref.tensor_exponent(_np(small))
    assert ctx.qesgd_status() == 0


def test_more_than_2_to_31_elements():
    rows, cols = 70_000, 40_000                      # 2.8e9 elements
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("too little memory")
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    for r in (0, 127, 53_000, 69_900):
        x[r:r + 100] = torch.randn((min(100, rows - r), cols), generator=torch.Generator(device="cuda").manual_seed(r), device="cuda")
    ctx, fmt = G.ctx(), qesgd.FP4_MX
    held = qesgd.alloc_fp4(rows, cols, fmt, "cuda")
    held_t = qesgd.alloc_fp4(cols, rows, fmt, "cuda")
    ctx.qesgd_fp4_quantize(x, qesgd.BF16, rows, cols, cols, fmt, None, qesgd.ROUND_STOCHASTIC, 3, 1, 2, *held, *held_t)
    back = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    ctx.qesgd_fp4_dequantize(*held, rows, cols, fmt, None, back, qesgd.BF16, cols)
    for r in (0, 53_000, 69_900):
        part = _np(x[r:r + 100])
        codes, byte, _ = ref.quantize(part, fmt)
        index = (np.arange(r, r + part.shape[0])[:, None] * cols + np.arange(cols)[None, :])      # cols is a multiple of 32
        q = np.abs(part) / np.repeat(ref.E8M0[byte], 32, 1)[:, :cols]
        low = np.searchsorted(ref.GRID, q, side="right") - 1
        gap = np.where(low < 7, ref.GRID[np.minimum(low + 1, 7)] - ref.GRID[low], 1.0)
        up = (ref.draws(index, 3, 1, 2) + 0.5) / 65536.0 < (q - ref.GRID[low]) / gap
        want = np.sign(part) * ref.GRID[np.minimum(low + up, 7)] * np.repeat(ref.E8M0[byte], 32, 1)[:, :cols]
        assert (_np(back[r:r + 100]) == want).all()
    # the transpose: its last rows against those of a matrix of their own (rounded to nearest, the draws being others)
    ctx.qesgd_fp4_quantize(x, qesgd.BF16, rows, cols, cols, fmt, None, qesgd.ROUND_NEAREST, 0, 0, 0, None, None, *held_t)
    got = torch.empty((cols, rows), dtype=torch.bfloat16, device="cuda")
    ctx.qesgd_fp4_dequantize(*held_t, cols, rows, fmt, None, got, qesgd.BF16, rows)
    part = _np(x[:, -40:].T)
    codes, byte, _ = ref.quantize(part, fmt)
    assert (_np(got[-40:]) == ref.values(codes, byte, fmt)).all()
    assert ctx.qesgd_status() == 0


def test_refused_calls_enqueue_nothing():
    ctx = G.ctx()
    n = ctx.qesgd_launch_count()
    x = torch.ones((4, 8), device="cuda")
    c = torch.full((4, 4), 3.0, device="cuda")
    codes, scales = qesgd.alloc_fp4(4, 8, qesgd.FP4_MX, "cuda")
    e = torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(qesgd.QesgdError):
        ctx.qesgd_fp4_quantize(x, qesgd.F32, 4, 8, 7, qesgd.FP4_MX, None, 0, 0, 0, 0, codes, scales)
    with pytest.raises(qesgd.QesgdError):
        ctx.qesgd_fp4_quantize(x, qesgd.F32, 4, 8, 8, qesgd.FP4_MX, e, 0, 0, 0, 0, codes, scales)
    with pytest.raises(qesgd.QesgdError):
        ctx.qesgd_fp4_matmul(codes, scales, None, codes, scales, None, 4, 4, 8, qesgd.FP4_MX, c, qesgd.F32, 3)
    with pytest.raises(qesgd.QesgdError):
        ctx.qesgd_orthogonalize(x, qesgd.F32, 4, 8, 8, 1, 0, 5, c, 8, 0, codes, 16)
    torch.cuda.synchronize()
    assert ctx.qesgd_launch_count() == n and (c == 3.0).all()


# ------------------------------------------------------------ used together ----
def test_a_round_on_a_weight_matrix():
    """Two workers each take one step of a linear least-squares layer with 4-bit products (forward, gradient of the
    inputs, gradient of the weight), encode the delta of their weight; the server averages the streams into a fresh
    update, makes it orthogonal and applies it.  Every part against 64 bits on what went into it."""
    T, I, O, K = 96, 160, 224, 2        # tokens, inputs, outputs, workers
    g = torch.Generator().manual_seed(0)
    W = (torch.randn((O, I), generator=g) * 0.1).cuda()
    ctx, fmt = G.ctx(), qesgd.FP4_NV
    assert ctx.qesgd_status() == 0
    w, _ = _quantize(W, I, fmt, "rc", dtype=qesgd.F32)            # for Y = X W^T and dX = dY W
    wv = [ref.values(*ref.quantize(v, fmt)[:2], fmt) for v in (_np(W), _np(W).T)]
    d, bucket, s, bits = O * I, 512, 127, 8
    codes, scales = qesgd.alloc_stream_buffers(K, d, bucket, bits, "cuda")
    locals_ = torch.empty((K, O, I), device="cuda")
    for k in range(K):
        X = torch.randn((T, I), generator=g).to(torch.bfloat16).cuda()
        target = torch.randn((T, O), generator=g).cuda()
        x, _ = _quantize(X, I, fmt, "rc", dtype=qesgd.BF16)
        xv = [ref.values(*ref.quantize(v, fmt)[:2], fmt) for v in (_np(X), _np(X).T)]
        Y = torch.empty((T, O), device="cuda")
        ctx.qesgd_fp4_matmul(*x["r"], None, *w["r"], None, T, O, I, fmt, Y, qesgd.F32, O)
        y = xv[0] @ wv[0].T
        assert (np.abs(_np(Y) - y) <= (I + 4) * 2.0 ** -23 * (np.abs(xv[0]) @ np.abs(wv[0]).T)).all()
        dY = (Y - target) / T
        e = torch.empty(1, dtype=torch.int32, device="cuda")
        ctx.qesgd_fp4_tensor_exponent(dY, qesgd.F32, T, O, O, e)
        t = ref.tensor_exponent(_np(dY))
        assert int(e) == t
        gq, _ = _quantize(dY, O, fmt, "rc", 5, k, 1, exponent=e, dtype=qesgd.F32)
        gv = [ref.values(*ref.quantize(v, fmt, t, 5, k, 1)[:2], fmt, t) for v in (_np(dY), _np(dY).T)]
        dX, dW = torch.empty((T, I), device="cuda"), torch.zeros((O, I), device="cuda")
        ctx.qesgd_fp4_matmul(*gq["r"], e, *w["c"], None, T, I, O, fmt, dX, qesgd.F32, I)
        ctx.qesgd_fp4_matmul(*gq["c"], e, *x["c"], None, O, I, T, fmt, dW, qesgd.F32, I, 1)
        assert (np.abs(_np(dX) - gv[0] @ wv[1].T) <= (O + 4) * 2.0 ** -23 * (np.abs(gv[0]) @ np.abs(wv[1]).T)).all()
        assert (np.abs(_np(dW) - gv[1] @ xv[1].T) <= (T + 4) * 2.0 ** -23 * (np.abs(gv[1]) @ np.abs(xv[1]).T)).all()
        # the gradient of the loss |X W^T - target|^2 / 2T at the quantised operands, against a difference quotient: the loss is
        # quadratic along any direction, so central differences are exact
        D = np.random.default_rng(k).standard_normal((O, I))
        loss = lambda w_: 0.5 / T * np.sum((xv[0] @ w_.T - _np(target)) ** 2)  # noqa: E731
        slope = (loss(wv[0] + 1e-3 * D) - loss(wv[0] - 1e-3 * D)) / 2e-3
        exact = ((xv[0] @ wv[0].T - _np(target)) / T).T @ xv[0]
        assert abs(slope - np.sum(exact * D)) <= 1e-6 * abs(slope)
        # stochastic and nearest 4-bit operands leave the direction of the exact gradient
        cos = np.sum(_np(dW) * exact) / np.linalg.norm(_np(dW)) / np.linalg.norm(exact)
        assert cos > 0.95
        locals_[k] = W - 0.5 * dW
    ctx.qesgd_encode_batch(locals_.view(K, d), d, W, d, K, bucket, s, bits, qesgd.SCALE_NORM, 7, 0, 0, codes, codes.stride(0),
                           scales, scales.stride(0))
    update = torch.zeros((O, I), device="cuda")
    ctx.qesgd_decode_average_apply(update, d, K, codes, codes.stride(0), scales, scales.stride(0), bucket, s, bits)
    O_ = _orthogonalize(update[None], qesgd.F32, O, I)[0]
    want = ref.orthogonalize(_np(update))
    assert np.linalg.norm(_np(O_) - want) <= ORTHO_TOLERANCE * np.linalg.norm(want)
    sv = np.linalg.svd(_np(O_), compute_uv=False)
    assert sv[0] < 1.3 and np.mean(sv > 0.5) > 0.9
    # the step goes downhill to first order: it has a positive product with the averaged delta
    assert float((O_.float() * update).sum()) > 0
    assert ctx.qesgd_status() == 0
