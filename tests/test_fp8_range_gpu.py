"""The 8-bit path at the lower end of the number range: subnormal numbers are numbers, in scales' products, sums, norms and outputs.

Tolerances.  Those of test_fp8_gpu.py, and below 2^-126, where a rounding is off by half a step of 2^-149 whatever the value, that many half
steps more."""
import pytest
import torch

from paper_2410_09615_b200 import binding as K

pytestmark = pytest.mark.gpu

E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
HALF = {E4: 2.0 ** -4, E5: 2.0 ** -3}
HALF_STEP = {E4: 2.0 ** -10, E5: 2.0 ** -17}
TINY = 2.0 ** -126
HALF32 = 2.0 ** -150                    # half a step of a subnormal binary32 number
HALF16 = 2.0 ** -134                    # of a subnormal bf16 number

# (one of each kernel of the layer: clusters of one and of eight CTAs, single CTAs and pairs on token tiles, both ways out)
SIZES = [(1, 8192, 64), (3, 128, 300), (16, 1040, 1030), (30, 8192, 300), (64, 6000, 520), (64, 1728, 5121), (100, 2752, 520), (230, 2064, 4100), (600, 1728, 5120), (1030, 384, 2001)]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def product(Xs, Ws, d_out):
    """Each token's and row's product of scales, rounded to binary32 as the contract has it (on the CPU, which keeps subnormal numbers)."""
    w = Ws.cpu().repeat_interleave(128, 0)[:d_out]
    return (Xs.cpu().unsqueeze(1) * w.unsqueeze(0)).double().cuda()                   # [b, d_out, groups]


def sums(Xq, Wq, s, absolute=False):
    """Sum over the groups of a product of scales times the group's inner product, in 64 bits."""
    X, W = Xq.double(), Wq.double()
    if absolute:
        X, W = X.abs(), W.abs()
    Y = torch.zeros(X.shape[0], W.shape[0], dtype=torch.float64, device="cuda")
    for g in range(s.shape[2]):
        Y += s[:, :, g] * (X[:, 128 * g:128 * g + 128] @ W[:, 128 * g:128 * g + 128].T)
    return Y


@pytest.mark.parametrize("low", [-124, -126, -130, -136])
@pytest.mark.parametrize("b, d_in, d_out", SIZES)
def test_linear_keeps_subnormal_products_of_scales(b, d_in, d_out, low):
    """Whole numbers, and scales that are powers of two whose product is 2^low to 2^(low - 6): multiples of 2^-142, all below 2^24 of them, so every
    product and sum is exact, and Y is rounded once."""
    g = gen(b - low)
    Xq = torch.randint(-2, 3, (b, d_in), generator=g, device="cuda").float().to(E4)
    Wq = torch.randint(-2, 3, (d_out, d_in), generator=g, device="cuda").float().to(E4)
    G, N = -(-d_in // 128), -(-d_out // 128)
    ones = lambda r: torch.ones((r, G), dtype=torch.float64, device="cuda")       # noqa: E731
    Xs = torch.ldexp(ones(b), -60 - torch.randint(0, 4, (b, G), generator=g, device="cuda")).float()
    Ws = torch.ldexp(ones(N), low + 60 - torch.randint(0, 4, (N, G), generator=g, device="cuda")).float()
    s = product(Xs, Ws, d_out)
    Y = K.slim_linear_fwd_fp8(Xq, Xs, Wq, Ws)
    ref = sums(Xq, Wq, s)
    assert ref.abs().max() > 0 and torch.equal(Y.double().cpu(), ref.float().cpu().bfloat16().double())


@pytest.mark.parametrize("x, w", [(E4, E4), (E5, E5)])
@pytest.mark.parametrize("b, d_in, d_out", SIZES)
def test_linear_with_products_of_scales_around_the_smallest_normal_number(b, d_in, d_out, x, w):
    g = gen(b)
    Xq, Wq = torch.randn((b, d_in), generator=g, device="cuda").mul(40).to(x), torch.randn((d_out, d_in), generator=g, device="cuda").mul(40).to(w)
    G, N = -(-d_in // 128), -(-d_out // 128)
    Xs = torch.exp2(-60 - 10 * torch.rand((b, G), generator=g, device="cuda"))
    Ws = torch.exp2(-60 - 14 * torch.rand((N, G), generator=g, device="cuda"))
    s = product(Xs, Ws, d_out)
    ref, size = sums(Xq, Wq, s), sums(Xq, Wq, s, True)
    off = (128 + 2 + G) * 2.0 ** -23
    Y = K.slim_linear_fwd_fp8(Xq, Xs, Wq, Ws)
    assert ((Y.double() - ref).abs() <= (2.0 ** -8 + off) * ref.abs() + off * size + HALF16 + (G + 8) * HALF32).all()
    assert (Y != 0).float().mean() > 0.9
