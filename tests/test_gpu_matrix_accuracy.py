"""How near the orthogonalised update is to the exact one, whatever its spectrum."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_1901_03040_b200 import qesgd                     # noqa: E402
from tests import gpu_helpers as G                          # noqa: E402

# What five usual steps may be off, as a share of the result's 2-norm.
#   The result's rounding to bf16: an element is off by at most 2^-8 of it, 0.425 * 2^-8 = 1.66e-3 in the mean of squares over
#   mantissas spread evenly over their logarithm (uniform error within a unit, whose share of the value falls from 2^-8 to 2^-9).
#   A and B off their diagonals are kept in fp16, three bits finer: r = 2.08e-4 in the same mean.  With p(s) / s = a + b s^2 + c s^4,
#   an error of A enters X' as (b + 2 c s^2) s^2 / (p(s) / s) of it, at most 1.33 times (s^2 = 0.8), one of B as
#   (b s^2 + c s^4) / (p(s) / s), at most 4.4 times (s^2 = 1.17): 4.6 r = 9.6e-4 a step, and sqrt(5) of that, 2.2e-3, for
#   five steps of independent roundings.
#   Together sqrt(1.66^2 + 2.2^2) = 2.75e-3.
ROUNDING = 0.425 * 2.0 ** -8
STEP = 4.6 * 0.425 * 2.0 ** -11
WIDE_TOLERANCE = float(np.hypot(ROUNDING, np.sqrt(5.0) * STEP))


def _orthogonalize(x, steps=5, **coefficients):
    batch, rows, cols = x.shape
    need = qesgd.orthogonalize_workspace(rows, cols, batch)
    work = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")           # NaN in every type
    out = torch.empty((batch, rows, cols), dtype=torch.bfloat16, device="cuda")
    G.ctx().qesgd_orthogonalize(x, qesgd.F32, rows, cols, x.stride(1), batch, x.stride(0) if batch > 1 else 0, steps, out, cols,
                                rows * cols, work, need, **coefficients)
    return out


def _exact(x, steps=5, a=3.4445, b=-4.7750, c=2.0315):
    x = x.double()
    turned = x.shape[1] > x.shape[2]
    x = x.mT if turned else x
    x = x / torch.linalg.matrix_norm(x, keepdim=True)
    for _ in range(steps):
        g = x @ x.mT
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.mT if turned else x


def _off(got, want):
    norm = torch.linalg.matrix_norm
    return (norm(got.double() - want) / norm(want)).tolist()


def _strong(rows, cols, strong, rest, seed):
    """`strong` directions over noise `rest` times as large."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, strong), generator=g) @ torch.randn((strong, cols), generator=g) / strong ** 0.5
    return (x + rest * torch.randn((rows, cols), generator=g)).cuda()


def _spectra(rows, cols):
    k = min(rows, cols)
    return torch.stack([_strong(rows, cols, r, rest, 7 * i + r)
                        for r in sorted({1, 4, 16, k // 4, k // 2}) if 0 < 2 * r <= k
                        for i, rest in enumerate((1e-1, 1e-2, 1e-3, 1e-5))])


@pytest.mark.parametrize("rows,cols", [(16, 64), (1000, 16), (32, 512), (48, 48), (64, 256), (64, 1000), (100, 1000), (128, 128), (700, 120),
                                       (128, 4096)])
def test_far_singular_values_in_one_kernel(rows, cols):
    x = _spectra(rows, cols)
    for part in x.split(8):
        part = part.contiguous()
        off = _off(_orthogonalize(part), _exact(part))
        assert max(off) <= WIDE_TOLERANCE, off
    assert G.ctx().qesgd_status() == 0


@pytest.mark.parametrize("rows,cols", [(2, 3), (4, 16), (8, 8), (100, 8), (12, 300)])
def test_far_singular_values_of_few_rows(rows, cols):
    """So few elements that the result's rounding may be near its most, 2^-8, in the ones that count."""
    x = _spectra(rows, cols)
    off = _off(_orthogonalize(x), _exact(x))
    assert max(off) <= 2.0 ** -8 + np.sqrt(5.0) * STEP, off
    assert G.ctx().qesgd_status() == 0


@pytest.mark.parametrize("rows,cols", [(129, 130), (129, 1000), (1000, 200), (256, 512), (300, 1500), (500, 500), (512, 512), (512, 2048), (700, 700)])
def test_far_singular_values_in_products_of_their_own(rows, cols):
    for x in _spectra(rows, cols):
        off = _off(_orthogonalize(x[None]), _exact(x[None]))
        assert max(off) <= WIDE_TOLERANCE, off
    x = _spectra(rows, cols)[::5][:4].contiguous()                # and as a batch
    off = _off(_orthogonalize(x), _exact(x))
    assert max(off) <= WIDE_TOLERANCE, off
    assert G.ctx().qesgd_status() == 0


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 9])
@pytest.mark.parametrize("rows,cols", [(60, 200), (140, 400), (600, 700)])
def test_far_singular_values_after_other_numbers_of_steps(rows, cols, steps):
    """X's second term and the products that take it, from the first step to behind the third."""
    x = _strong(rows, cols, 4, 1e-3, steps)[None]
    off = _off(_orthogonalize(x, steps), _exact(x, steps))
    assert max(off) <= float(np.hypot(ROUNDING, np.sqrt(steps) * STEP)), off


@pytest.mark.parametrize("steps", [3, 4])
@pytest.mark.parametrize("rows,cols", [(100, 300), (128, 2000), (129, 200), (300, 200), (200, 1030), (140, 4200)])
def test_what_is_kept_between_steps_is_cut_off(rows, cols, steps):
    """One element to a row, each in a column of its own: rows stay apart, and x' = x (a + b x^2 + c x^4) for each, cut off at
    65504 / 256 between steps.  With a, b, c > 0 a relative error of x enters x' at most fivefold, and x^4 is that of the
    fp16 operand, whose rounding, 2^-11, counts four times: e' <= 5 e + 2^-9.  Cut off after the second or third step, where it is
    exact, an element has the last step's error, or the last two's: 6 * 2^-9, and 2^-8 for the result's rounding."""
    k = min(rows, cols)
    v = torch.linspace(0.5, 1.5, k, dtype=torch.float32)
    x = torch.zeros((2, rows, cols))
    at = torch.arange(k) * (cols // k if rows <= cols else 1)
    if rows <= cols:
        x[:, torch.arange(k), at] = v
    else:
        x[:, torch.arange(k) * (rows // k), torch.arange(k)] = v
    a, b, c = 16.0, 32.0, 32.0
    got = _orthogonalize(x.cuda(), steps, a=a, b=b, c=c).cpu().double()
    kept = x.double() / torch.linalg.matrix_norm(x.double(), keepdim=True)
    most = 65504.0 / 256.0
    cut = torch.zeros_like(kept, dtype=torch.bool)
    for step in range(steps):
        kept = kept * (a + b * kept ** 2 + c * kept ** 4)
        if step + 1 < steps:
            cut |= kept.abs() > most
            kept = kept.clamp(-most, most)
    assert cut.any()
    off = ((got - kept).abs() / kept.abs().clamp_min(1e-30))[cut]
    assert float(off.max()) <= 6 * 2.0 ** -9 + 2.0 ** -8, float(off.max())
    assert (got[x == 0] == 0).all()
    assert G.ctx().qesgd_status() == 0


@pytest.mark.parametrize("rows,cols", [(5, 700), (700, 5), (10, 256), (20, 2000), (40, 4500), (100, 4000), (4000, 128), (140, 9000), (9000, 140)])
def test_nearly_orthogonal_rows(rows, cols):
    """Few long rows are nearly orthogonal to begin with, so A and B are nearly diagonal, and their diagonals are kept in 32 bits:
    the errors of a step (STEP above) count only by the share of A and B that lies off them; a diagonal element itself is a sum
    over a row of squares rounded to fp16, whose errors average to 2 / sqrt(row's length) of one.  Beside that, the rounding of this very
    result to bf16.  (Diagonals in fp16, too, would end 1.8e-3 to 3.3e-3 off here, X without its second term 1.8e-3, at bounds of
    1.68e-3 to 1.9e-3.)"""
    for seed in range(3):
        g = torch.Generator().manual_seed(seed)
        x = torch.randn((1, rows, cols), generator=g).cuda()
        want = _exact(x)
        y = x[0].double() if rows < cols else x[0].double().T
        y, share = y / y.norm(), 0.0
        for _ in range(5):
            A = y @ y.T
            B = -4.7750 * A + 2.0315 * A @ A
            share = max([share] + [float((m - torch.diag(m.diagonal())).norm() / m.norm()) for m in (A, B)])
            y = 3.4445 * y + B @ y
        rounding = _off(want.to(torch.bfloat16), want)[0]
        errors = np.sqrt(5.0) * STEP * (share + 2.0 / max(rows, cols) ** 0.5)
        off = _off(_orthogonalize(x), want)[0]
        assert off <= np.hypot(rounding, errors), (seed, off, rounding, errors)


def _shared_errors(m, n, r):
    """What fp16 operands leave of five steps on an m x n matrix, m <= n, with r equal singular values s and nothing else, as a share
    of the result, before its rounding: X = s U V^T, q = p(s) / s, all errors independent with mean square (rho x value)^2.
      A = X X^T of rounded X: U^T dA U has r^2 entries of 2 (rho s^2)^2 r / (m n): 2 rho^2 r^2 / (m n) of |A|^2.
      A's rounding off the diagonal: r^2 / m^2 rho^2 of |A|^2 between the U, rho^2 elsewhere.  B's: the same of |B|^2.
    An error of A enters X' by (b + 2 c s^2) s^2 / q, one of B by (b s^2 + c s^4) / q.  Between the U, later steps enlarge it by
    g = s p'(s) / p(s) each; elsewhere it turns U, which p leaves as it is (by 1)."""
    a, b, c, rho, s, steps = 3.4445, -4.7750, 2.0315, 0.425 * 2.0 ** -11, r ** -0.5, []
    for _ in range(5):
        q = a + b * s ** 2 + c * s ** 4
        steps.append(((b + 2 * c * s ** 2) * s ** 2 / q, (b * s ** 2 + c * s ** 4) / q, (a + 3 * b * s ** 2 + 5 * c * s ** 4) / q))
        s *= q
    square = 0.0
    for i, (by_a, by_b, _) in enumerate(steps):
        g2 = float(np.prod([g for _, _, g in steps[i + 1:]])) ** 2
        square += (by_a * rho) ** 2 * (g2 * (2 * r * r / (m * n) + r * r / (m * m)) + 1) + (by_b * rho) ** 2 * (g2 * r * r / (m * m) + 1)
    return square ** 0.5


@pytest.mark.parametrize("rows,cols", [(4, 4), (8, 8), (16, 16), (16, 64), (24, 30), (32, 32), (40, 40), (300, 64), (100, 300), (128, 128), (200, 200), (300, 520), (640, 640)])
def test_equal_strong_singular_values(rows, cols):
    """r equal singular values, the rest 10^-3 of them.  What the r share is enlarged by the steps that follow, s p'(s) / p(s)
    each, up to 18 times in all, which WIDE_TOLERANCE leaves out; _shared_errors has it."""
    k = min(rows, cols)
    xs, bounds = [], []
    for i, strong in enumerate(sorted({k // 8, k // 4, k // 2, k - k // 8, k} - {0})):
        g = torch.Generator(device="cuda").manual_seed(i)
        u = torch.linalg.qr(torch.randn((rows, k), generator=g, device="cuda", dtype=torch.float64))[0]
        v = torch.linalg.qr(torch.randn((cols, k), generator=g, device="cuda", dtype=torch.float64))[0]
        s = torch.full((k,), 1e-3, device="cuda", dtype=torch.float64)
        s[:strong] = 1.0
        xs.append(((u * s) @ v.T).float())
        want = _exact(xs[-1][None])
        # r^2 errors make up the shared ones: their mean square is off by sqrt(2 / r^2) of itself, three times that at most
        bounds.append(np.hypot(_off(want.to(torch.bfloat16), want)[0], (1.0 + 2.1 / strong) * _shared_errors(k, max(rows, cols), strong)))
    x = torch.stack(xs)
    off = _off(_orthogonalize(x), _exact(x))
    if k < 512:
        assert (np.array(off) <= np.array(bounds)).all(), (off, bounds)
    if k >= 64:
        assert max(off) <= WIDE_TOLERANCE, off
    assert G.ctx().qesgd_status() == 0
