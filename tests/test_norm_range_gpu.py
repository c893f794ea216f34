"""The norm at the lower end of the number range: subnormal numbers are numbers, in eps, sums, mean squares and outputs.

Tolerances.  Those of test_fp8_gpu.py, and below 2^-126, where a rounding is off by half a step of 2^-149 whatever the value, that many half
steps more."""
import pytest
import torch

from paper_2410_09615_b200 import binding as K

pytestmark = pytest.mark.gpu

E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
TOP = {E4: 448.0, E5: 57344.0}
HALF = {E4: 2.0 ** -4, E5: 2.0 ** -3}
HALF_STEP = {E4: 2.0 ** -10, E5: 2.0 ** -17}
TINY = 2.0 ** -126
HALF32 = 2.0 ** -150                    # half a step of a subnormal binary32 number
HALF16 = 2.0 ** -134                    # of a subnormal bf16 number
# (as in test_fp8_gpu.py: fewer than 100 roundings in a chain of a row's sum, of which the square root halves, and four more)
NORM_OFF = (100 / 2 + 4) * 2.0 ** -23
ROWS = [(1, 16), (5, 272), (3, 4096), (200, 2048), (2, 16400)]


def small(b, d, seed, std):
    """bf16, made in 64 bits on the CPU: subnormal numbers among them."""
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((b, d), generator=g, dtype=torch.float64) * std).float().bfloat16().cuda()


def exact(X, gamma, eps, R):
    """(h, y, mean square + eps) in 64 bits; eps as binary32 has it."""
    h = X.double() + (0 if R is None else R.double())
    eps = float(torch.tensor(eps, dtype=torch.float64).float().double())
    m = (h * h).mean(1, keepdim=True) + eps
    return h, h / m.sqrt() * gamma.double(), m


def check(X, gamma, eps, R, off=0.0, steps=0.0):
    """Both forms; y may be off by `off` of its value more than by NORM_OFF, and by `steps`."""
    h, y, _ = exact(X, gamma, eps, R)
    off = off + NORM_OFF
    Y, H = K.slim_rmsnorm(X, gamma, eps, R)
    assert ((Y.double() - y).abs() <= (2.0 ** -8 + off) * y.abs() + steps + HALF16).all()
    assert H is None or torch.equal(H.double().cpu(), h.cpu().float().bfloat16().double())
    for dtype in (E4, E5):
        codes, scales, H8 = K.slim_rmsnorm_fp8(X, gamma, eps, R, dtype=dtype)
        assert H8 is None or torch.equal(H8.double(), H.double())
        by = scales.double().repeat_interleave(128, 1)[:, :X.shape[1]]
        pad = torch.zeros(X.shape[0], scales.shape[1] * 128, dtype=torch.float64, device="cuda")
        pad[:, :X.shape[1]] = y
        s = (pad.view(X.shape[0], -1, 128).abs().amax(2) / TOP[dtype]).clamp_min(TINY)
        assert ((scales.double() - s).abs() <= (off + 2.0 ** -23) * s + steps).all()
        assert ((codes.double() * by - y).abs() <= (HALF[dtype] + 2 * off) * y.abs() + HALF_STEP[dtype] * by * (1 + off) + steps).all()
    return Y


def gamma_of(d):
    return (1 + 0.1 * torch.randn(d, generator=torch.Generator().manual_seed(1))).bfloat16().cuda()


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("b, d", ROWS)
def test_subnormal_inputs(b, d, residual):
    """h of 2^-130: the mean square is eps, 2^-100, and y about 2^-80."""
    Y = check(small(b, d, d, 2.0 ** -130), gamma_of(d), 2.0 ** -100, small(b, d, d + 1, 2.0 ** -130) if residual else None)
    assert (Y != 0).any()


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("b, d", ROWS)
def test_subnormal_outputs(b, d, residual):
    """y of about 2^-130: rounded once behind each of two products, the first error times gamma."""
    gamma = gamma_of(d)
    Y = check(small(b, d, d, 2.0 ** -70), gamma, 2.0 ** 120, small(b, d, d + 1, 2.0 ** -70) if residual else None,
              steps=(1 + float(gamma.abs().max())) * HALF32)
    assert (Y != 0).any()


@pytest.mark.parametrize("eps", [2.0 ** -149, 1e-40, 2.0 ** -126])
@pytest.mark.parametrize("b, d", ROWS)
def test_rows_of_zeros_and_the_smallest_eps(b, d, eps):
    gamma = gamma_of(d)
    X = small(b, d, d, 1.0)
    X[0] = 0.0
    Y = check(X, gamma, eps, None)
    assert (Y[0] == 0).all()
    codes, scales, _ = K.slim_rmsnorm_fp8(X, gamma, eps)
    assert (codes[0].float() == 0).all() and (scales[0] == TINY).all()


@pytest.mark.parametrize("eps", [2.0 ** -149, 2.0 ** -130])
@pytest.mark.parametrize("b, d", ROWS)
def test_subnormal_mean_squares(b, d, eps):
    """h of 2^-65: every one of the sum's d additions is off by half a step at most, the mean by another, and it plus eps by none."""
    X, gamma = small(b, d, d, 2.0 ** -65), gamma_of(d)
    _, _, m = exact(X, gamma, eps, None)
    check(X, gamma, eps, None, off=float(2 * HALF32 / m.min()))


@pytest.mark.parametrize("eps", [2.0 ** -149, 2.0 ** -100, 2.0 ** -65, 2.0 ** -64])
@pytest.mark.parametrize("d", [16, 2048, 16400])
def test_sums_on_both_sides_of_where_they_are_scaled(d, eps):
    """Rows whose sums of squares go from 2^-72 to 2^-56 (scaled are those below 2^-64, where eps is below it too)."""
    X = small(17, d, d, 1.0).double()
    X = (X * torch.exp2(torch.arange(17, device="cuda") / 2.0 - 36).unsqueeze(1) / (X * X).sum(1, keepdim=True).sqrt()).float().bfloat16()
    check(X, gamma_of(d), eps, None)
