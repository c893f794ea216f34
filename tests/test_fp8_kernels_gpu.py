"""Every kernel of the 8-bit layer, by its name: clusters of each size, and token tiles with more of them than CTAs or pairs, where the rings, the
accumulators and the way out are used again.  Rows of Y that are and are not a multiple of 16 bytes leave by two ways.

Tolerances: those of test_fp8_gpu.py."""
import pytest
import torch

from paper_2410_09615_b200 import binding as K

pytestmark = pytest.mark.gpu

E4 = torch.float8_e4m3fn
TILES = {"cluster_16": (16, 128), "cluster_32": (32, 128), "cluster_64": (64, 128), "cluster_128": (128, 128), "rows_32": (128, 32), "rows_64": (128, 64),
         "rows_128": (128, 128), "pair_128": (256, 128), "pair_256": (256, 256)}

# tokens, columns, rows, kernel, CTAs of a cluster
CLUSTERS = [(8, 512, 300, "cluster_16", 1), (16, 1040, 1030, "cluster_16", 2), (16, 2064, 3000, "cluster_16", 4), (11, 8192, 301, "cluster_16", 8),
            (30, 656, 260, "cluster_32", 1), (25, 2064, 9001, "cluster_32", 2), (30, 2064, 3000, "cluster_32", 4), (30, 8192, 300, "cluster_32", 8),
            (64, 656, 11008, "cluster_32", 1), (64, 5120, 13824, "cluster_64", 1), (50, 4096, 11008, "cluster_64", 1), (64, 5120, 13001, "cluster_64", 1),
            (64, 6000, 9000, "cluster_64", 2), (333, 8192, 1030, "cluster_128", 4)]
# with more tiles than SMs or pairs
TOKENS = [(4096, 128, 272, "rows_32"), (4096, 128, 271, "rows_32"), (1000, 128, 1168, "rows_32"), (1000, 128, 1167, "rows_32"), (20000, 1168, 32, "rows_32"),
          (20000, 1168, 31, "rows_32"), (4000, 512, 520, "rows_64"), (4000, 512, 513, "rows_64"), (12000, 1168, 160, "rows_64"),
          (100, 4096, 30000, "rows_128"), (100, 4096, 29999, "rows_128"), (3000, 400, 1001, "rows_128"), (520, 1728, 8200, "pair_128"),
          (520, 1728, 8201, "pair_128"), (1100, 512, 20000, "pair_256"), (1100, 512, 19999, "pair_256")]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def spread(v, rows, cols):
    return v.double().repeat_interleave(128, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def check(b, d_in, d_out, kernel, ctas):
    """Normal operands with a scale of its own for every group, against 64 bits; then whole numbers and powers of two, where every sum is exact."""
    g = gen(b + d_in)
    G, N = -(-d_in // 128), -(-d_out // 128)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    Xq, Wq = torch.randn((b, d_in), generator=g, device="cuda").mul(40).to(E4), torch.randn((d_out, d_in), generator=g, device="cuda").mul(40).to(E4)
    Xs, Ws = torch.rand((b, G), generator=g, device="cuda") + 0.01, torch.rand((N, G), generator=g, device="cuda") + 0.01
    Y = K.slim_linear_fwd_fp8(Xq, Xs, Wq, Ws, status=status)
    assert K.slim_last_fp8_kernel() == (kernel, ctas) and K.slim_last_token_tile() == TILES[kernel][0] and K.slim_last_launch_count() == 1
    X, W = Xq.double() * Xs.double().repeat_interleave(128, 1)[:, :d_in], Wq.double() * spread(Ws, d_out, d_in)
    ref, size = X @ W.T, X.abs() @ W.abs().T
    off = (128 + 2 + G) * 2.0 ** -23
    assert ((Y.double() - ref).abs() <= (2.0 ** -8 + off) * ref.abs() + off * size).all()
    assert all(torch.equal(Y, K.slim_linear_fwd_fp8(Xq, Xs, Wq, Ws, status=status)) for _ in range(5))
    Xq, Wq = (torch.randint(-2, 3, (n, d_in), generator=g, device="cuda").float().to(E4) for n in (b, d_out))
    Xs, Ws = (2.0 ** torch.randint(-2, 3, (n, G), generator=g, device="cuda").float() for n in (b, N))
    ref = (Xq.double() * Xs.double().repeat_interleave(128, 1)[:, :d_in]) @ (Wq.double() * spread(Ws, d_out, d_in)).T
    assert torch.equal(K.slim_linear_fwd_fp8(Xq, Xs, Wq, Ws, status=status), ref.bfloat16()) and int(status) == 0


@pytest.mark.parametrize("b, d_in, d_out, kernel, ctas", CLUSTERS)
def test_clusters(b, d_in, d_out, kernel, ctas):
    check(b, d_in, d_out, kernel, ctas)


@pytest.mark.parametrize("b, d_in, d_out, kernel", TOKENS)
def test_several_tiles(b, d_in, d_out, kernel):
    tokens, rows = TILES[kernel]
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert -(-b // tokens) * -(-d_out // rows) > (sms // 2 if "pair" in kernel else sms)
    check(b, d_in, d_out, kernel, 1)


def test_the_query_is_of_the_last_call():
    """And of the calling thread."""
    import threading
    X, W = torch.randn((4, 128), device="cuda").bfloat16(), torch.randn((64, 128), device="cuda")
    ops = K.slim_quant_fp8(X) + K.slim_pack_fp8(W)
    assert K.slim_last_fp8_kernel() == ("none", 1)
    K.slim_linear_fwd_fp8(*ops)
    assert K.slim_last_fp8_kernel() == ("cluster_16", 1)
    seen = []
    other = threading.Thread(target=lambda: seen.append(K.slim_last_fp8_kernel()))
    other.start(), other.join()
    assert seen == [("none", 1)]
    K.slim_quant_fp8(X)
    assert K.slim_last_fp8_kernel() == ("none", 1)
