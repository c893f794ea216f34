"""The 8-bit path against plain implementations: quantisers bit for bit, norm and linear layer against 64 bits.

Tolerances.  A rounding is off by half a step at most, eps / 2 of the value: bf16 2^-8, fp32 2^-24, e4m3 2^-4, e5m2 2^-3 (below the
smallest normal code half of the smallest step: 2^-10 and 2^-17).  A sum of n terms in binary32, in whatever order, is off by less than
n 2^-23 times the sum of the magnitudes, also where every addition truncates instead of rounding."""
import pytest
import torch

from paper_2410_09615_b200 import binding as K

pytestmark = pytest.mark.gpu

E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
TOP = {E4: 448.0, E5: 57344.0}
HALF = {E4: 2.0 ** -4, E5: 2.0 ** -3}
HALF_STEP = {E4: 2.0 ** -10, E5: 2.0 ** -17}
TINY = 2.0 ** -126
INF, NAN = float("inf"), float("nan")


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rows(b, d, seed=0, std=1.0):
    g = gen(seed)
    loud = torch.where(torch.rand(d, generator=g, device="cuda") < 0.02, 30.0, 1.0)
    return (torch.randn((b, d), generator=g, device="cuda") * loud * std).bfloat16()


def spread(v, by):
    """[rows, groups] -> a value for each of `v`'s elements; by: rows that share a scale."""
    return v.repeat_interleave(by, 0).repeat_interleave(128, 1)


def quantised(v, dtype, by=1):
    """The definition, step by step in binary32 on the CPU: (codes, scales)."""
    v = v.float().cpu()
    r, c = v.shape
    pad = torch.zeros(-(-r // by) * by, -(-c // 128) * 128)
    pad[:r, :c] = v
    scale = pad.view(pad.shape[0] // by, by, -1, 128).abs().amax((1, 3)) / TOP[dtype]
    scale = torch.where(scale < TINY, torch.full_like(scale, TINY), scale)
    inv = 1.0 / scale
    return (pad * spread(inv, by)).clamp(-TOP[dtype], TOP[dtype])[:r, :c].to(dtype), scale


def same_bits(a, b):
    a, b = a.cpu(), b.cpu()
    if a.dtype in (E4, E5):
        a, b = a.float(), b.float()
    return a.shape == b.shape and torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a[~torch.isnan(a)], b[~torch.isnan(b)])


def awkward(v):
    """Zeros, ties, tiny and huge groups among ordinary ones."""
    v = v.clone()
    v[0, :min(128, v.shape[1])] = 0.0
    if v.shape[0] > 2:
        v[1] *= 1e-38                       # scales at their lower end, subnormal values
        v[2] *= 1e36
    if v.shape[0] > 4:
        v[3] = torch.arange(v.shape[1], device=v.device) % 97 * 0.0625          # many ties
        v[4] = -1.75
    return v


# ---------------------------------------------------------------- quantisers
@pytest.mark.parametrize("dtype", [E4, E5])
@pytest.mark.parametrize("b, d", [(1, 16), (1, 4096), (3, 144), (5, 128), (7, 1008), (64, 1136), (333, 1728), (17, 28672), (2048, 512)])
def test_quant_is_the_definition(b, d, dtype):
    X = awkward(rows(b, d, b + d))
    codes, scales = K.slim_quant_fp8(X, dtype)
    assert codes.dtype == dtype and scales.shape == (b, -(-d // 128))
    c, s = quantised(X, dtype)
    assert same_bits(scales, s) and same_bits(codes, c)


@pytest.mark.parametrize("dtype", [E4, E5])
@pytest.mark.parametrize("type_", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d_out, d_in", [(1, 16), (128, 128), (5, 400), (129, 144), (300, 1040), (511, 2048), (1000, 272)])
def test_pack_is_the_definition(d_out, d_in, type_, dtype):
    W = awkward(torch.randn((d_out, d_in), generator=gen(d_out), device="cuda") * 0.02).to(type_)
    codes, scales = K.slim_pack_fp8(W, dtype)
    assert codes.dtype == dtype and scales.shape == (-(-d_out // 128), -(-d_in // 128))
    c, s = quantised(W, dtype, 128)
    assert same_bits(scales, s) and same_bits(codes, c)


@pytest.mark.parametrize("dtype", [E4, E5])
def test_quant_passes_nan_and_infinity_on(dtype):
    X = rows(4, 512, 3)
    X[1, 130], X[2, 300], X[3, 400] = NAN, INF, -INF
    codes, scales = K.slim_quant_fp8(X, dtype)
    c, s = quantised(X, dtype)
    assert same_bits(scales, s) and same_bits(codes, c)
    assert torch.isnan(scales[1, 1]) and torch.isinf(scales[2, 2]) and torch.isfinite(scales[0]).all()
    value = codes.float() * scales.repeat_interleave(128, 1)
    assert torch.isnan(value[1, 128:256]).all() and torch.isnan(value[2, 256:384]).all() and torch.isnan(value[3, 384:]).all()
    assert torch.isfinite(value[1, :128]).all()


# ---------------------------------------------------------------- norm
def norm64(X, gamma, eps, residual):
    h = X.double() + (0 if residual is None else residual.double())
    return h, h / ((h * h).mean(1, keepdim=True) + eps).sqrt() * gamma.double()


# (a row's squares are added by up to 32 a thread, then over 32 lanes and 32 warps: fewer than 100 roundings in a chain; the square root
# halves what they come to; four more roundings to y)
NORM_OFF = (100 / 2 + 4) * 2.0 ** -23


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("b, d", [(1, 16), (1, 4096), (2, 128), (3, 272), (5, 2048), (4, 2064), (600, 5120), (3, 8192), (2, 16384), (2, 16400), (1, 28672), (3, 32768)])
def test_norm_against_64_bits(b, d, residual):
    X, gamma = rows(b, d, d), (1 + 0.1 * torch.randn(d, generator=gen(1), device="cuda")).bfloat16()
    R = rows(b, d, d + 1, 2.0) if residual else None
    h, y = norm64(X, gamma, 1e-5, R)
    Y, H = K.slim_rmsnorm(X, gamma, 1e-5, R)
    assert Y.dtype == torch.bfloat16 and ((Y.double() - y).abs() <= (2.0 ** -8 + NORM_OFF) * y.abs()).all()
    if residual:
        assert torch.equal(H, (X.float() + R.float()).bfloat16())
    else:
        assert H is None
    for dtype in (E4, E5):
        codes, scales, H8 = K.slim_rmsnorm_fp8(X, gamma, 1e-5, R, dtype=dtype)
        assert (H8 is None) == (not residual) and (H8 is None or torch.equal(H8, H))
        pad = torch.zeros(b, scales.shape[1] * 128, dtype=torch.float64, device="cuda")
        pad[:, :d] = y
        s = pad.view(b, -1, 128).abs().amax(2) / TOP[dtype]
        assert ((scales.double() - s).abs() <= (NORM_OFF + 2.0 ** -23) * s).all()
        by = scales.double().repeat_interleave(128, 1)[:, :d]
        assert ((codes.double() * by - y).abs() <= (HALF[dtype] + 2 * NORM_OFF) * y.abs() + HALF_STEP[dtype] * by * (1 + NORM_OFF)).all()
        # the largest of a group is the format's largest number
        assert (codes.float().abs().amax(1) == TOP[dtype]).all()


def test_norm_writes_the_sum_in_place():
    X, R, gamma = rows(33, 1040, 1), rows(33, 1040, 2), torch.ones(1040, device="cuda").bfloat16()
    Y, H = K.slim_rmsnorm(X, gamma, 1e-6, R)
    X2, R2 = X.clone(), R.clone()
    Y2, H2 = K.slim_rmsnorm(X, gamma, 1e-6, R2, H=R2)
    assert H2.data_ptr() == R2.data_ptr() and torch.equal(R2, H) and torch.equal(Y2, Y)
    out = torch.empty_like(Y)
    Y3, H3 = K.slim_rmsnorm(X2, gamma, 1e-6, R, H=X2, Y=out)
    assert Y3.data_ptr() == out.data_ptr() and torch.equal(X2, H) and torch.equal(out, Y)
    codes, scales, H4 = K.slim_rmsnorm_fp8(X, gamma, 1e-6, R)
    R2 = R.clone()
    codes2, scales2, _ = K.slim_rmsnorm_fp8(X, gamma, 1e-6, R2, H=R2)
    assert torch.equal(R2, H4) and same_bits(codes, codes2) and torch.equal(scales, scales2)
    Y5, H5 = K.slim_rmsnorm(X, gamma, 1e-6, None, H=torch.empty_like(X))      # without a residual: a copy of X
    assert torch.equal(H5, X)


def test_norm_rows_are_independent():
    X, gamma = rows(6, 512, 4), torch.ones(512, device="cuda").bfloat16()
    clean, _ = K.slim_rmsnorm(X, gamma, 1e-5)
    X[1], X[2, 7], X[4, 500] = 0.0, NAN, INF
    Y, _ = K.slim_rmsnorm(X, gamma, 1e-5)
    assert (Y[1] == 0).all() and torch.isnan(Y[2]).all() and torch.equal(Y[[0, 3, 5]], clean[[0, 3, 5]])
    codes, scales, _ = K.slim_rmsnorm_fp8(X, gamma, 1e-5)
    assert (codes[1].float() == 0).all() and (scales[1] == TINY).all()
    assert torch.isnan(scales[2]).all() and torch.isnan(codes[2].float()).all()
    assert torch.isfinite(codes[[0, 1, 3, 5]].float()).all()


# ---------------------------------------------------------------- the linear layer
def operands(b, d_in, d_out, seed, x=E4, w=E4):
    Xq, Xs = K.slim_quant_fp8(rows(b, d_in, seed), x)
    Wq, Ws = K.slim_pack_fp8(torch.randn((d_out, d_in), generator=gen(seed + 1), device="cuda") * 0.02, w)
    return Xq, Xs, Wq, Ws


def check_linear(Xq, Xs, Wq, Ws, Y, at=None):
    """Y's rows `at` (all) against 64 bits."""
    if at is not None:
        Xq, Xs, Y = Xq[at], Xs[at], Y[at]
    d_out, d_in = Wq.shape
    X = Xq.double() * Xs.double().repeat_interleave(128, 1)[:, :d_in]
    W = Wq.double() * spread(Ws.double(), 128)[:d_out, :d_in]
    ref, size = X @ W.T, X.abs() @ W.abs().T
    # 128 terms of a group, its scales' product and the groups
    off = (128 + 2 + Xs.shape[1]) * 2.0 ** -23
    bad = (Y.double() - ref).abs() > (2.0 ** -8 + off) * ref.abs() + off * size
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), Y[bad][:4].tolist(), ref[bad][:4].tolist())


SIZES = [(1, 16, 1), (1, 128, 16), (1, 4096, 512), (2, 144, 130), (3, 4096, 4096), (5, 1728, 640), (8, 512, 512), (16, 5120, 5120), (16, 272, 128),
         (17, 2048, 1000), (31, 1040, 257), (33, 4096, 1024), (64, 1376, 4096), (65, 512, 384), (100, 2752, 520), (127, 384, 2048), (128, 4096, 256),
         (129, 1024, 1024), (200, 3456, 1360), (255, 256, 512), (257, 640, 256), (333, 2048, 2048), (512, 1728, 1288), (600, 1728, 5120), (777, 1152, 999),
         (1024, 4096, 1024), (1500, 528, 4096), (2049, 512, 513), (4096, 256, 768)]


@pytest.mark.parametrize("b, d_in, d_out", SIZES)
def test_linear_against_64_bits(b, d_in, d_out):
    o = operands(b, d_in, d_out, b + d_in)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    Y = K.slim_linear_fwd_fp8(*o, status=status)
    assert Y.shape == (b, d_out) and Y.dtype == torch.bfloat16 and K.slim_last_launch_count() == 1
    check_linear(*o, Y)
    assert torch.equal(Y, K.slim_linear_fwd_fp8(*o, status=status)) and int(status) == 0


# Each kernel with several tiles a CTA or pair, columns that end inside a block, four or eight groups, and rows of Y that are and are not a
# multiple of 16 bytes; the tokens that its tile has.
KERNELS = [(16, 1040, 1030, 16), (16, 8192, 300, 16), (9, 2064, 9000, 16), (30, 656, 260, 32), (30, 8192, 300, 32), (25, 2064, 9001, 32),
           (64, 6000, 9000, 64), (50, 400, 100, 32), (128, 8192, 16, 32), (200, 8192, 1030, 32), (100, 14208, 4480, 64), (2100, 5120, 100, 32),
           (70, 144, 16, 128), (520, 144, 100, 128), (333, 8192, 1030, 128), (130, 8208, 1930, 128), (64, 1728, 5121, 32), (230, 2064, 4100, 128),
           (3000, 400, 1001, 128), (200, 2064, 5120, 256), (3000, 2064, 513, 256), (520, 1728, 8200, 256), (200, 1040, 9999, 256),
           (1500, 1040, 2050, 256), (520, 1728, 4100, 256), (2100, 3600, 1030, 256), (1100, 512, 20000, 256)]


@pytest.mark.parametrize("b, d_in, d_out, tokens", KERNELS)
def test_every_kernel_of_the_linear_layer(b, d_in, d_out, tokens):
    o = operands(b, d_in, d_out, 3 * b + d_in)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    Y = K.slim_linear_fwd_fp8(*o, status=status)
    assert K.slim_last_token_tile() == tokens and K.slim_last_launch_count() == 1
    check_linear(*o, Y)
    for _ in range(5):
        assert torch.equal(Y, K.slim_linear_fwd_fp8(*o, status=status))
    assert int(status) == 0


@pytest.mark.parametrize("x, w", [(E4, E5), (E5, E4), (E5, E5)])
@pytest.mark.parametrize("b, d_in, d_out", [(1, 1024, 400), (16, 656, 512), (64, 2048, 320), (130, 1040, 640), (700, 1728, 1100)])
def test_linear_formats(b, d_in, d_out, x, w):
    o = operands(b, d_in, d_out, 7, x, w)
    check_linear(*o, K.slim_linear_fwd_fp8(*o))


@pytest.mark.parametrize("b, d_in, d_out", [(1, 256, 300), (4, 8192, 64), (16, 1424, 700), (60, 2048, 1030), (150, 640, 520), (300, 1040, 777), (1030, 384, 2000)])
def test_linear_places_every_element(b, d_in, d_out):
    """Small whole numbers and scales that are powers of two, another one for every row, block and group: every product and sum is exact."""
    g = gen(b)
    Xq = torch.randint(-2, 3, (b, d_in), generator=g, device="cuda").float().to(E4)
    Wq = torch.randint(-2, 3, (d_out, d_in), generator=g, device="cuda").float().to(E4)
    G, N = -(-d_in // 128), -(-d_out // 128)
    Xs = 2.0 ** torch.randint(-2, 3, (b, G), generator=g, device="cuda").float()
    Ws = 2.0 ** torch.randint(-2, 3, (N, G), generator=g, device="cuda").float()
    X, W = Xq.double() * Xs.double().repeat_interleave(128, 1)[:, :d_in], Wq.double() * spread(Ws.double(), 128)[:d_out, :d_in]
    assert torch.equal(K.slim_linear_fwd_fp8(Xq, Xs, Wq, Ws), (X @ W.T).bfloat16())


@pytest.mark.parametrize("b", [1, 20, 90, 260])
def test_linear_one_element_each(b):
    """One activation a token, one weight a row: each lands where it belongs."""
    d_in, d_out = 1040, 270
    m, n = torch.arange(b, device="cuda"), torch.arange(d_out, device="cuda")
    k = (n * 37 + 5) % d_in
    W = torch.zeros(d_out, d_in, device="cuda")
    W[n, k] = ((n % 7) + 1).float()
    X = torch.zeros(b, d_in, device="cuda")
    X[m, k[m % d_out]] = 2.0
    ones = lambda r: torch.ones(r, -(-d_in // 128), device="cuda")       # noqa: E731
    Y = K.slim_linear_fwd_fp8(X.to(E4), ones(b), W.to(E4), ones(-(-d_out // 128)))
    assert torch.equal(Y, (X.double() @ W.double().T).bfloat16())


@pytest.mark.parametrize("b", [2, 40, 100, 400])
def test_linear_keeps_nan_and_infinity_in_their_rows(b):
    d_in, d_out = 656, 400
    X, W = rows(b, d_in, 9), (torch.randn((d_out, d_in), generator=gen(3), device="cuda") * 0.02).bfloat16()
    clean = K.slim_linear_fwd_fp8(*K.slim_quant_fp8(X), *K.slim_pack_fp8(W))
    X[1, 650], X[0, 3] = NAN, INF
    W[130, 5] = NAN                                              # its block's 128 rows
    Y = K.slim_linear_fwd_fp8(*K.slim_quant_fp8(X), *K.slim_pack_fp8(W))
    assert torch.isnan(Y[:2]).all() and torch.isnan(Y[:, 128:256]).all()
    keep = torch.ones(d_out, dtype=torch.bool)
    keep[128:256] = False
    assert torch.equal(Y[2:, keep], clean[2:, keep])


@pytest.mark.parametrize("b, lo, hi", [(40, 1, 14), (300, 3, 290)])
def test_linear_on_rows_of_a_larger_batch(b, lo, hi):
    """Rows of a batch: scales of 4-byte alignment; the output is a part of a larger tensor, and what lies around it stays."""
    Xq, Xs, Wq, Ws = operands(b, 640, 136, 2)
    whole = K.slim_linear_fwd_fp8(Xq, Xs, Wq, Ws)
    out = torch.full((b, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    K.slim_linear_fwd_fp8(Xq[lo:hi], Xs[lo:hi], Wq, Ws, Y=out[lo:hi])
    check_linear(Xq, Xs, Wq, Ws, out, slice(lo, hi))
    assert (out[:lo] == 7).all() and (out[hi:] == 7).all()
    assert torch.equal(out[lo:hi], whole[lo:hi]) or (out[lo:hi].float() - whole[lo:hi].float()).abs().max() <= 2.0 ** -7 * whole.abs().max()


@pytest.mark.parametrize("b, d_out", [(1, 999), (16, 1001), (70, 131), (300, 777)])
def test_linear_writes_its_rows_only(b, d_out):
    o = operands(b, 512, d_out, 4)
    flat = torch.full((b * d_out + 4096,), 3.0, dtype=torch.bfloat16, device="cuda")
    Y = flat[:b * d_out].view(b, d_out)
    K.slim_linear_fwd_fp8(*o, Y=Y)
    check_linear(*o, Y)
    assert (flat[b * d_out:] == 3).all()


def test_linear_on_another_stream_and_two_at_once():
    shapes = [(16, 2048, 4096), (64, 4096, 1024), (200, 2048, 2048), (1000, 1024, 2048)]
    ops = [operands(*s, 11) for s in shapes]
    refs = [K.slim_linear_fwd_fp8(*o) for o in ops]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ops]
    outs = [[] for _ in ops]
    for _ in range(10):
        for i, (s, o) in enumerate(zip(streams, ops)):
            with torch.cuda.stream(s):
                outs[i].append(K.slim_linear_fwd_fp8(*o))
    torch.cuda.synchronize()
    for r, got in zip(refs, outs):
        assert all(torch.equal(r, y) for y in got)


def test_a_block_of_a_model_captured_and_replayed():
    """norm -> 8-bit layer -> quantiser -> 8-bit layer, and norm -> 4-bit layer, as a decoder's MLP uses them: eager, captured, replayed on
    new inputs."""
    d, inner, b = 1024, 2736, 24
    gamma = (1 + 0.1 * torch.randn(d, generator=gen(1), device="cuda")).bfloat16()
    up, down = torch.randn((inner, d), generator=gen(2), device="cuda") * 0.02, torch.randn((d, inner), generator=gen(3), device="cuda") * 0.02
    U, D = K.slim_pack_fp8(up), K.slim_pack_fp8(down)
    codes, sa, _, _ = K.slim_quant(torch.randn((512, d), generator=gen(4), device="cuda") * 0.02)
    vals, meta = K.slim_pack(codes, K.slim_mask_top2(codes))
    s, ws = float(sa[0]), K.new_workspace(b, 512, d, 0)
    x, res = rows(b, d, 5), rows(b, d, 6, 2.0)

    def block():
        Xq, Xs, H = K.slim_rmsnorm_fp8(x, gamma, 1e-5, res)
        mid = K.slim_linear_fwd_fp8(Xq, Xs, *U)
        out = K.slim_linear_fwd_fp8(*K.slim_quant_fp8(mid), *D)
        Y, H2 = K.slim_rmsnorm(out, gamma, 1e-5, H)
        return Xq, Xs, H, mid, out, Y, H2, K.slim_linear_fwd(Y, vals, meta, s, None, None, workspace=ws)

    def check(got):
        Xq, Xs, H, mid, out, Y, H2, last = got
        assert torch.equal(H, (x.float() + res.float()).bfloat16())
        check_linear(Xq, Xs, *U, mid)
        check_linear(*K.slim_quant_fp8(mid), *D, out)
        assert torch.equal(H2, (out.float() + H.float()).bfloat16())
        y = norm64(out, gamma, 1e-5, H)[1]
        assert ((Y.double() - y).abs() <= (2.0 ** -8 + NORM_OFF) * y.abs()).all()
        assert torch.equal(last, K.slim_linear_fwd(Y, vals, meta, s, None, None))

    check(block())
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        block()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = block()
    for seed in (8, 9):
        x.copy_(rows(b, d, seed)), res.copy_(rows(b, d, seed + 10, 2.0))
        graph.replay()
        torch.cuda.synchronize()
        check(got)


def test_more_elements_than_32_bits_count():
    b, d = (1 << 32) // 16384 + 300, 16384
    X = torch.zeros((b, d), dtype=torch.bfloat16, device="cuda")
    tail = rows(300, d, 1)
    X[-300:] = tail
    codes, scales = K.slim_quant_fp8(X)
    c, s = quantised(tail, E4)
    assert same_bits(scales[-300:], s) and same_bits(codes[-300:], c)
    W = torch.randn((48, d), generator=gen(2), device="cuda") * 0.02
    Wq, Ws = K.slim_pack_fp8(W)
    Y = K.slim_linear_fwd_fp8(codes, scales, Wq, Ws)
    check_linear(codes, scales, Wq, Ws, Y, slice(b - 300, b))
    assert (Y[:-300] == 0).all()
    del Y, codes, scales
    gamma = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    codes, scales, _ = K.slim_rmsnorm_fp8(X, gamma, 1e-5)
    one, one_s, _ = K.slim_rmsnorm_fp8(tail, gamma, 1e-5)
    assert same_bits(codes[-300:], one) and same_bits(scales[-300:], one_s)


# ---------------------------------------------------------------- refusals
def test_shapes_that_do_not_match_are_refused():
    Xq, Xs, Wq, Ws = operands(4, 256, 128, 0)
    for bad in ([Xq, Xs[:, :1].contiguous(), Wq, Ws], [Xq, Xs, Wq[:, :128].contiguous(), Ws], [Xq, Xs, Wq, Ws[:, :1].contiguous()], [Xq[:3], Xs, Wq, Ws]):
        with pytest.raises(ValueError):
            K.slim_linear_fwd_fp8(*bad)
    with pytest.raises(ValueError):
        K.slim_linear_fwd_fp8(Xq, Xs, Wq, Ws, Y=torch.empty(4, 127, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(TypeError):
        K.slim_linear_fwd_fp8(Xq, Xs, Wq, Ws, Y=torch.empty(4, 128, dtype=torch.float32, device="cuda"))
    with pytest.raises(TypeError):
        K.slim_linear_fwd_fp8(Xq[:, ::2], Xs, Wq, Ws)
    with pytest.raises(TypeError):
        K.slim_linear_fwd_fp8(Xq, Xs, Wq, Ws, status=torch.zeros(1, device="cuda"))
    X = rows(4, 256)
    gamma = torch.ones(256, dtype=torch.bfloat16, device="cuda")
    for call in (K.slim_rmsnorm, K.slim_rmsnorm_fp8):
        with pytest.raises(ValueError):
            call(X, gamma[:128].contiguous(), 1e-5)
        with pytest.raises(ValueError):
            call(X, gamma, 1e-5, X[:2])
        with pytest.raises(TypeError):
            call(X.float(), gamma, 1e-5)
        with pytest.raises(K.SlimError):
            call(X, gamma, 0.0)
        with pytest.raises(K.SlimError):
            call(X[:0], gamma, 1e-5)
        with pytest.raises(K.SlimError):
            call(X[:, :8].contiguous(), gamma[:8].contiguous(), 1e-5)
    for call in (K.slim_quant_fp8, K.slim_pack_fp8):
        with pytest.raises(TypeError):
            call(X, torch.int8)
        with pytest.raises(K.SlimError):
            call(X[:, :24].contiguous())
        with pytest.raises(K.SlimError):
            call(X[:0])
    with pytest.raises(K.SlimError):
        K.slim_linear_fwd_fp8(Xq[:0], Xs[:0], Wq, Ws)


def test_bad_tensors_leave_the_device_usable():
    with pytest.raises(TypeError):
        K.slim_linear_fwd_fp8(None, None, None, None)
    o = operands(4, 256, 128, 0)
    check_linear(*o, K.slim_linear_fwd_fp8(*o))


def test_first_call_of_a_process_in_a_capture():
    """What a call sets up once per device does not disturb a capture."""
    import os
    import subprocess
    import sys
    code = (
        "import torch\n"
        "from paper_2410_09615_b200 import binding as K\n"
        "X = torch.randn(200, 512, device='cuda').bfloat16(); W = torch.randn(300, 512, device='cuda')\n"
        "gamma = torch.ones(512, device='cuda').bfloat16()\n"
        "K.native(); torch.cuda.synchronize()\n"
        "def f():\n"
        "    Wp = K.slim_pack_fp8(W)\n"
        "    return [K.slim_linear_fwd_fp8(*K.slim_rmsnorm_fp8(X[:b], gamma, 1e-5, X[:b])[:2], *Wp) for b in (1, 20, 50, 200)]\n"
        "g = torch.cuda.CUDAGraph()\n"
        "with torch.cuda.graph(g):\n"
        "    got = f()\n"
        "g.replay(); torch.cuda.synchronize()\n"
        "assert all(torch.equal(a, b) for a, b in zip(got, f())); print('ok')\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stderr[-2000:]


def test_calls_on_two_threads():
    import threading
    o = [operands(b, 1040, 700, b) for b in (8, 300)]
    refs = [K.slim_linear_fwd_fp8(*x) for x in o]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(100):
                if not torch.equal(K.slim_linear_fwd_fp8(*o[i]), refs[i]):
                    bad.append(i)

    threads = [threading.Thread(target=work, args=(i % 2,)) for i in range(4)]
    [t.start() for t in threads], [t.join() for t in threads]
    assert not bad


def test_other_threads_run_during_a_call(tmp_path):
    """The calls give the interpreter to other threads: a stand-in for the library's function returns only when another thread has run
    (or, with an error, after a second)."""
    import ctypes
    import subprocess
    import threading
    import time
    src, so = tmp_path / "stall.c", tmp_path / "stall.so"
    src.write_text("#include <time.h>\nvolatile int go = 0;\nint stall(void) {\n    struct timespec nap = {0, 1000000};\n"
                   "    for (int i = 0; i < 1000; ++i) { if (go) return 0; nanosleep(&nap, 0); }\n    return 6;\n}\n")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", str(src), "-o", str(so)], check=True)
    stand_in = ctypes.CDLL(str(so))
    go = ctypes.c_int.in_dll(stand_in, "go")
    addr = lambda f: ctypes.cast(f, ctypes.c_void_p).value       # noqa: E731
    own = [addr(getattr(K.lib(), n)) for n in ("slim_rmsnorm", "slim_rmsnorm_fp8", "slim_quant_fp8", "slim_pack_fp8", "slim_linear_fwd_fp8")]
    o, X, gamma = operands(2, 128, 128, 0), rows(2, 128), torch.ones(128, device="cuda").bfloat16()
    native = K.native()
    try:
        native.bind_fp8(*[addr(stand_in.stall)] * 5)
        for call in (lambda: K.slim_rmsnorm(X, gamma, 1e-5), lambda: K.slim_rmsnorm_fp8(X, gamma, 1e-5), lambda: K.slim_quant_fp8(X),
                     lambda: K.slim_pack_fp8(X), lambda: K.slim_linear_fwd_fp8(*o)):
            go.value = 0
            other = threading.Thread(target=lambda: (time.sleep(0.02), setattr(go, "value", 1)))
            other.start()
            try:
                call()                                           # raises where the other thread could not run
            finally:
                other.join()
    finally:
        native.bind_fp8(*own)
    check_linear(*o, K.slim_linear_fwd_fp8(*o))
