"""What the matrix operators refuse, and their sizes: host code that runs before anything touches a device, so no GPU is
needed.  A block of zeros stands in for a context: a call that is let through ends with a CUDA error here."""
import ctypes as C

import pytest

BIG = (1 << 40) + 1


@pytest.fixture(scope="module")
def qesgd():
    from paper_1901_03040_b200 import build
    build.build()
    from paper_1901_03040_b200 import qesgd as mod
    return mod


@pytest.fixture(scope="module")
def ctx(qesgd):
    import torch
    if torch.cuda.is_available():
        pytest.skip("would run accepted calls on made-up addresses")
    return C.cast(C.create_string_buffer(4096), C.c_void_p)


def test_sizes(qesgd):
    assert [qesgd.fp4_row_bytes(c) for c in (0, 1, 32, 33, 4096)] == [0, 16, 16, 32, 2048]
    assert qesgd.fp4_row_bytes(qesgd.MAX_MATRIX_SIDE + 1) == 0
    assert qesgd.fp4_scale_bytes(1, 1, qesgd.FP4_MX) == qesgd.fp4_scale_bytes(128, 128, qesgd.FP4_MX) == 512
    assert qesgd.fp4_scale_bytes(129, 129, qesgd.FP4_MX) == 2048
    assert qesgd.fp4_scale_bytes(128, 129, qesgd.FP4_NV) == 3 * 512
    assert qesgd.fp4_scale_bytes(0, 5, qesgd.FP4_NV) == qesgd.fp4_scale_bytes(5, 0, qesgd.FP4_NV) == 0
    assert qesgd.fp4_scale_bytes(5, 5, 2) == 0
    assert qesgd.orthogonalize_workspace(0, 5) == qesgd.orthogonalize_workspace(5, 5, 0) == 0
    assert qesgd.orthogonalize_workspace(65537, 5) == qesgd.orthogonalize_workspace(5, 5, 4097) == 0
    assert qesgd.orthogonalize_workspace(64, 256) >= 4 * 64 * 256 * 2
    assert qesgd.orthogonalize_workspace(64, 256) == qesgd.orthogonalize_workspace(256, 64)


def _call(qesgd, name, order, good, **change):
    args = [C.c_void_p(v) if n in PTRS and v is not None else v for n, v in [(n, {**good, **change}[n]) for n in order]]
    return getattr(qesgd.lib, name)(*args)


PTRS = {"x", "e", "codes", "scales", "codes_t", "scales_t", "out", "a", "sa", "b", "sb", "ta", "tb", "c", "work"}
QUANTIZE = "ctx x dtype rows cols ldx format e rounding seed worker epoch codes scales codes_t scales_t".split()
GOOD_QUANTIZE = dict(x=4096, dtype=0, rows=10, cols=40, ldx=40, format=1, e=4096, rounding=1, seed=1, worker=0, epoch=0,
                     codes=4096, scales=4096, codes_t=4096, scales_t=4096)


@pytest.mark.parametrize("change", [
    dict(dtype=3), dict(format=2), dict(rounding=2), dict(x=None), dict(x=4098), dict(x=4097, dtype=1), dict(ldx=39),
    dict(ldx=BIG), dict(rows=0x7FFFFF01), dict(cols=0x7FFFFF01), dict(codes=None), dict(scales=None), dict(codes_t=None),
    dict(scales_t=None), dict(codes=None, scales=None, codes_t=None, scales_t=None), dict(codes=4104), dict(scales=4104),
    dict(codes_t=4104), dict(scales_t=4104), dict(e=4098), dict(format=0)])
def test_quantize_refuses(qesgd, ctx, change):
    assert _call(qesgd, "qesgd_fp4_quantize", QUANTIZE, dict(GOOD_QUANTIZE, ctx=ctx), **change) == qesgd.EINVAL


@pytest.mark.parametrize("change", [dict(), dict(codes=None, scales=None), dict(codes_t=None, scales_t=None), dict(e=None),
                                    dict(format=0, e=None), dict(x=4098, dtype=2), dict(ldx=41)])
def test_quantize_takes(qesgd, ctx, change):
    assert _call(qesgd, "qesgd_fp4_quantize", QUANTIZE, dict(GOOD_QUANTIZE, ctx=ctx), **change) == qesgd.ECUDA


@pytest.mark.parametrize("change", [dict(rows=0), dict(cols=0), dict(rows=0, x=None, codes=None, scales=None)])
def test_quantize_of_nothing(qesgd, ctx, change):
    assert _call(qesgd, "qesgd_fp4_quantize", QUANTIZE, dict(GOOD_QUANTIZE, ctx=ctx), **change) == qesgd.OK


def test_null_contexts(qesgd):
    lib = qesgd.lib
    assert _call(qesgd, "qesgd_fp4_quantize", QUANTIZE, dict(GOOD_QUANTIZE, ctx=None)) == qesgd.EINVAL
    assert _call(qesgd, "qesgd_fp4_matmul", MATMUL, dict(GOOD_MATMUL, ctx=None)) == qesgd.EINVAL
    assert _call(qesgd, "qesgd_orthogonalize", ORTHO, dict(GOOD_ORTHO, ctx=None)) == qesgd.EINVAL
    assert lib.qesgd_fp4_tensor_exponent(None, None, 0, 1, 1, 1, None) == qesgd.EINVAL
    assert lib.qesgd_fp4_dequantize(None, None, None, 1, 1, 0, None, None, 0, 1) == qesgd.EINVAL


DEQUANTIZE = "ctx codes scales rows cols format e out dtype ldo".split()
GOOD_DEQUANTIZE = dict(codes=4096, scales=4096, rows=10, cols=40, format=1, e=None, out=4096, dtype=1, ldo=40)


@pytest.mark.parametrize("change,want", [
    (dict(), "ECUDA"), (dict(codes=None), "EINVAL"), (dict(scales=None), "EINVAL"), (dict(codes=4100), "EINVAL"),
    (dict(out=None), "EINVAL"), (dict(out=4097), "EINVAL"), (dict(ldo=39), "EINVAL"), (dict(format=2), "EINVAL"),
    (dict(dtype=3), "EINVAL"), (dict(format=0, e=4096), "EINVAL"), (dict(rows=0), "OK"), (dict(cols=0), "OK")])
def test_dequantize_arguments(qesgd, ctx, change, want):
    assert _call(qesgd, "qesgd_fp4_dequantize", DEQUANTIZE, dict(GOOD_DEQUANTIZE, ctx=ctx), **change) == getattr(qesgd, want)


EXPONENT = "ctx x dtype rows cols ldx out".split()
GOOD_EXPONENT = dict(x=4096, dtype=0, rows=10, cols=40, ldx=40, out=4096)


@pytest.mark.parametrize("change,want", [
    (dict(), "ECUDA"), (dict(x=None), "EINVAL"), (dict(out=None), "EINVAL"), (dict(out=4098), "EINVAL"),
    (dict(ldx=39), "EINVAL"), (dict(dtype=3), "EINVAL"), (dict(x=4098), "EINVAL"), (dict(rows=0), "OK"), (dict(cols=0), "OK")])
def test_tensor_exponent_arguments(qesgd, ctx, change, want):
    assert _call(qesgd, "qesgd_fp4_tensor_exponent", EXPONENT, dict(GOOD_EXPONENT, ctx=ctx), **change) == getattr(qesgd, want)


MATMUL = "ctx a sa ta b sb tb M N K format c dtype ldc accumulate".split()
GOOD_MATMUL = dict(a=4096, sa=4096, ta=None, b=4096, sb=4096, tb=4096, M=10, N=20, K=30, format=1, c=4096, dtype=0, ldc=20,
                   accumulate=0)


@pytest.mark.parametrize("change,want", [
    (dict(), "ECUDA"), (dict(a=None), "EINVAL"), (dict(sa=None), "EINVAL"), (dict(b=None), "EINVAL"), (dict(sb=None), "EINVAL"),
    (dict(a=4104), "EINVAL"), (dict(sb=4104), "EINVAL"), (dict(c=None), "EINVAL"), (dict(c=4098), "EINVAL"),
    (dict(c=4098, dtype=1), "ECUDA"), (dict(ldc=19), "EINVAL"), (dict(format=2), "EINVAL"), (dict(format=0), "EINVAL"),
    (dict(dtype=3), "EINVAL"), (dict(ta=4097), "EINVAL"), (dict(M=0x7FFFFF01), "EINVAL"), (dict(K=0x7FFFFF01), "EINVAL"),
    (dict(M=0), "OK"), (dict(N=0, c=None), "OK"), (dict(K=0, accumulate=1), "OK"), (dict(K=0, a=None), "ECUDA")])
def test_matmul_arguments(qesgd, ctx, change, want):
    assert _call(qesgd, "qesgd_fp4_matmul", MATMUL, dict(GOOD_MATMUL, ctx=ctx), **change) == getattr(qesgd, want)


ORTHO = "ctx x dtype rows cols ldx batch xs steps p q r out ldo os work bytes".split()
GOOD_ORTHO = dict(x=4096, dtype=0, rows=10, cols=20, ldx=20, batch=2, xs=200, steps=5, p=3.4445, q=-4.775, r=2.0315, out=4096,
                  ldo=20, os=200, work=4096, bytes=1 << 20)


@pytest.mark.parametrize("change,want", [
    (dict(), "ECUDA"), (dict(x=None), "EINVAL"), (dict(x=4098), "EINVAL"), (dict(dtype=3), "EINVAL"), (dict(ldx=19), "EINVAL"),
    (dict(ldo=19), "EINVAL"), (dict(out=None), "EINVAL"), (dict(out=4097), "EINVAL"), (dict(xs=199), "EINVAL"),
    (dict(os=199), "EINVAL"), (dict(batch=1, xs=0, os=0), "ECUDA"), (dict(steps=0), "EINVAL"), (dict(steps=33), "EINVAL"),
    (dict(p=float("nan")), "EINVAL"), (dict(q=float("inf")), "EINVAL"), (dict(r=33.0), "EINVAL"), (dict(rows=65537), "EINVAL"),
    (dict(batch=4097), "EINVAL"), (dict(work=None), "EINVAL"), (dict(work=4096 + 128), "EINVAL"), (dict(bytes=100), "EINVAL"),
    (dict(rows=0), "OK"), (dict(cols=0), "OK"), (dict(batch=0), "OK")])
def test_orthogonalize_arguments(qesgd, ctx, change, want):
    assert _call(qesgd, "qesgd_orthogonalize", ORTHO, dict(GOOD_ORTHO, ctx=ctx), **change) == getattr(qesgd, want)


def test_the_smallest_workspace_is_the_stated_one(qesgd, ctx):
    need = qesgd.orthogonalize_workspace(10, 20, 2)
    good = dict(GOOD_ORTHO, ctx=ctx)
    assert _call(qesgd, "qesgd_orthogonalize", ORTHO, good, bytes=need) == qesgd.ECUDA
    assert _call(qesgd, "qesgd_orthogonalize", ORTHO, good, bytes=need - 1) == qesgd.EINVAL
