"""Workloads of the 8-bit path: what feeds a linear layer, and the layer whose weight is held in 8 bits.

Four kinds of case, as programs that use the library run them:

``linear``  one call of one layer whose weight was quantised once: Y = X W^T on 8-bit floating-point operands, the
            activations with a scale for each token and 128 columns, the weight with one for each block of 128 x 128.
``norm``    the step before a layer: the residual's addition, the root-mean-square norm and its output, in bf16 (for a layer of
            4-bit weights) or in 8 bits with scales (for one of 8-bit weights).
``quant``   activations that come from no norm (the input of an output or down projection) into 8 bits with scales.
``pack``    a layer's weight into 8 bits with scales, done once a layer.

Layer shapes are the LLaMA-2 7B / 13B / 70B linears, whole or as one rank's shard when the MLP's inner dimension is split
over 2, 4 or 8 GPUs, and any other width that is a multiple of 16.
"""
from __future__ import annotations

import math

import torch

own = False

_GROUP = 128
_FORMATS = {"e4m3": (torch.float8_e4m3fn, 448.0), "e5m2": (torch.float8_e5m2, 57344.0)}
_TINY = 2.0 ** -126                       # the smallest scale: the smallest normal binary32 number


_binding = None


def _library():
    global _binding
    if _binding is None:
        from paper_2410_09615_b200 import binding
        _binding = binding
    return _binding


def _linear(name, d_in, d_out, b, x="e4m3", w="e4m3"):
    return {"name": name, "op": "linear", "d_in": d_in, "d_out": d_out, "b": b, "x": x, "w": w}


def _norm(name, d, b, out, residual):
    return {"name": name, "op": "norm", "d": d, "b": b, "out": out, "residual": residual}


def listed():
    return [
        # the smallest layer the library is configured for, eight tokens
        _linear("linear_512x512_b8", 512, 512, 8),
        # one user's decode step: attention projection of the 7B model
        _linear("linear_4096x4096_b1", 4096, 4096, 1),
        # decode step of sixteen users: the largest layer of the 70B model (gate / up)
        _linear("linear_8192x28672_b16", 8192, 28672, 16),
        # decode step of a busy server, or a very short prompt: 64 tokens through the 13B gate / up layer
        _linear("linear_5120x13824_b64", 5120, 13824, 64),
        # a short prompt of no round length through a 70B attention projection, activations in the format of the wider range
        _linear("linear_8192x8192_b333_e5m2", 8192, 8192, 333, "e5m2"),
        # a prompt on one of eight GPUs that share the 13B model's MLP (down, an eighth of 13824): columns that end inside a block
        _linear("linear_1728x5120_b600", 1728, 5120, 600),
        # the largest: 4096 tokens through the 70B down projection
        _linear("linear_28672x8192_b4096", 28672, 8192, 4096),
        # one user's decode step: the norm before an 8-bit layer of the 7B model
        _norm("norm_4096_b1", 4096, 1, "e4m3", True),
        # a prompt of 4096 tokens: the norm before the 70B model's 8-bit layers
        _norm("norm_8192_b4096", 8192, 4096, "e4m3", True),
        # a prompt's first norm (no residual yet) before the 13B model's 4-bit layers
        _norm("norm_5120_b600_bf16", 5120, 600, "bf16", False),
        # a prompt's MLP activations before the 13B down projection
        {"name": "quant_13824_b2048", "op": "quant", "d": 13824, "b": 2048, "out": "e4m3"},
        # a weight on its way into 8 bits: 7B gate / up
        {"name": "pack_4096x11008", "op": "pack", "d_in": 4096, "d_out": 11008, "from": "bf16", "w": "e4m3"},
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _size(rng, lo, hi, step):
    return min(hi, max(lo, int(round(_log_uniform(rng, lo, hi) / step)) * step))


# (d_in, d_out) of the layers, and of one rank's shard of an MLP layer
_WHOLE = [(4096, 4096), (4096, 11008), (11008, 4096), (5120, 5120), (5120, 13824), (13824, 5120),
          (8192, 8192), (8192, 1024), (8192, 28672), (28672, 8192)]
_SHARDS = [(5504, 4096), (4096, 5504), (2752, 4096), (4096, 2752), (6912, 5120), (5120, 6912), (3456, 5120), (5120, 3456),
           (1728, 5120), (5120, 1728), (3584, 8192), (8192, 3584), (1376, 4096), (4096, 1376)]


def _tokens(rng, most=4096):
    """Half of the calls are decode steps, the others prompts and large batches."""
    return rng.randint(1, 16) if rng.random() < 0.4 else int(_log_uniform(rng, 17, most))


def draw(rng):
    kind = rng.random()
    width = rng.choice([4096, 5120, 8192, 11008, 13824, 28672, _size(rng, 512, 16384, 16)])
    if kind < 0.55:
        d_in, d_out = rng.choice([rng.choice(_WHOLE), rng.choice(_SHARDS), (_size(rng, 256, 8192, 16), _size(rng, 256, 8192, 16))])
        return {"op": "linear", "d_in": d_in, "d_out": d_out, "b": _tokens(rng), "x": "e5m2" if rng.random() < 0.2 else "e4m3",
                "w": "e5m2" if rng.random() < 0.1 else "e4m3"}
    if kind < 0.78:
        return {"op": "norm", "d": width, "b": _tokens(rng), "out": rng.choice(["e4m3", "e4m3", "e5m2", "bf16"]),
                "residual": rng.random() < 0.75}
    if kind < 0.9:
        return {"op": "quant", "d": width, "b": _tokens(rng), "out": rng.choice(["e4m3", "e4m3", "e5m2"])}
    d_in, d_out = rng.choice([rng.choice(_WHOLE), rng.choice(_SHARDS), (_size(rng, 512, 8192, 16), _size(rng, 512, 8192, 16))])
    return {"op": "pack", "d_in": d_in, "d_out": d_out, "from": rng.choice(["bf16", "f32"]), "w": rng.choice(["e4m3", "e4m3", "e5m2"])}


# ---- inputs

def _normal(shape, std, gen, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _activations(b, d, gen, std=1.0):
    """Rows of bf16 with a few channels far above the others, as a residual stream has them."""
    loud = torch.where(torch.rand(d, generator=gen, device="cuda") < 0.004, 20.0, 1.0)
    return (torch.randn((b, d), generator=gen, device="cuda") * loud * std).to(torch.bfloat16)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op = case["op"]
    if op == "norm":
        b, d = case["b"], case["d"]
        return {"case": case, "X": _activations(b, d, gen), "residual": _activations(b, d, gen, 2.0) if case["residual"] else None,
                "gamma": (1.0 + _normal((d,), 0.1, gen)).to(torch.bfloat16), "eps": 1e-5}
    if op == "quant":
        return {"case": case, "X": _activations(case["b"], case["d"], gen)}
    W = _normal((case["d_out"], case["d_in"]), 0.02, gen, torch.float32 if case.get("from") == "f32" else torch.bfloat16)
    if op == "pack":
        return {"case": case, "W": W}
    Wq, Ws = _quantised_blocks(W, case["w"])
    Xq, Xs = _quantised_rows(_activations(case["b"], case["d_in"], gen).float(), case["x"])
    return {"case": case, "Xq": Xq, "Xs": Xs, "Wq": Wq, "Ws": Ws}


# ---- plain forms

def _codes(v, scale, fmt):
    dtype, largest = _FORMATS[fmt]
    return (v * (1.0 / scale)).clamp(-largest, largest).to(dtype)


def _padded(v, dim):
    """Zeros behind the last column (or row) up to a multiple of 128."""
    short = -v.shape[dim] % _GROUP
    if short == 0:
        return v
    return torch.cat([v, v.new_zeros((v.shape[0], short) if dim == 1 else (short, v.shape[1]))], dim)


def _quantised_rows(v, fmt):
    """float32 [b, d] -> 8-bit codes [b, d] and scales [b, ceil(d / 128)]."""
    b, d = v.shape
    groups = _padded(v, 1).view(b, -1, _GROUP)
    scale = (groups.abs().amax(2) / _FORMATS[fmt][1]).clamp_min(_TINY)
    return _codes(groups, scale[:, :, None], fmt).view(b, -1)[:, :d].contiguous(), scale


def _quantised_blocks(W, fmt):
    """[d_out, d_in] -> 8-bit codes and scales [ceil(d_out / 128), ceil(d_in / 128)]."""
    d_out, d_in = W.shape
    v = _padded(_padded(W.float(), 1), 0)
    blocks = v.view(v.shape[0] // _GROUP, _GROUP, v.shape[1] // _GROUP, _GROUP)
    scale = (blocks.abs().amax((1, 3)) / _FORMATS[fmt][1]).clamp_min(_TINY)
    return _codes(blocks, scale[:, None, :, None], fmt).view(v.shape)[:d_out, :d_in].contiguous(), scale


def _normed(st, dtype):
    """(h, y) of the residual's addition and the norm, in `dtype`."""
    h = st["X"].to(dtype)
    if st["residual"] is not None:
        h = h + st["residual"].to(dtype)
    return h, h * torch.rsqrt(h.square().mean(1, keepdim=True) + st["eps"]) * st["gamma"].to(dtype)


def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        K = _library()
        if op == "linear":
            return K.slim_linear_fwd_fp8(st["Xq"], st["Xs"], st["Wq"], st["Ws"])
        if op == "quant":
            return K.slim_quant_fp8(st["X"], _FORMATS[case["out"]][0])
        if op == "pack":
            return K.slim_pack_fp8(st["W"], _FORMATS[case["w"]][0])
        if case["out"] == "bf16":
            return K.slim_rmsnorm(st["X"], st["gamma"], st["eps"], st["residual"])
        return K.slim_rmsnorm_fp8(st["X"], st["gamma"], st["eps"], st["residual"], dtype=_FORMATS[case["out"]][0])
    if op == "linear":
        d_out, d_in = st["Wq"].shape
        X = st["Xq"].float() * st["Xs"].repeat_interleave(_GROUP, 1)[:, :d_in]
        W = st["Wq"].float() * st["Ws"].repeat_interleave(_GROUP, 0)[:d_out].repeat_interleave(_GROUP, 1)[:, :d_in]
        return (X @ W.T).to(torch.bfloat16)
    if op == "quant":
        return _quantised_rows(st["X"].float(), case["out"])
    if op == "pack":
        return _quantised_blocks(st["W"], case["w"])
    h, y = _normed(st, torch.float32)
    H = None if st["residual"] is None else h.to(torch.bfloat16)
    if case["out"] == "bf16":
        return y.to(torch.bfloat16), H
    return (*_quantised_rows(y, case["out"]), H)


# ---- the same in 64 bits, from the definitions

def _row_scales(y, largest):
    """Scales of float64 rows, one group of columns after the other."""
    return torch.stack([y[:, k:k + _GROUP].abs().amax(1) for k in range(0, y.shape[1], _GROUP)], 1).div(largest).clamp_min(_TINY)


def exact(case, seed):
    """Codes are given as the values before their rounding to 8 bits.  Where that rounding alone moves them by 5% of their norm (two
    bits of significand), that value says nothing of them, and they have none."""
    st = prepare(case, seed)
    op = case["op"]
    if op == "linear":
        X, W, Xs, Ws = st["Xq"].double(), st["Wq"].double(), st["Xs"].double(), st["Ws"].double()
        block_of_row = torch.arange(W.shape[0], device="cuda") // _GROUP
        Y = torch.zeros((X.shape[0], W.shape[0]), dtype=torch.float64, device="cuda")
        for g in range(Xs.shape[1]):
            part = X[:, g * _GROUP:(g + 1) * _GROUP] @ W[:, g * _GROUP:(g + 1) * _GROUP].T
            Y += part.mul_(Xs[:, g, None]).mul_(Ws[block_of_row, g])
        return Y
    if op == "pack":
        W, largest = st["W"].double(), _FORMATS[case["w"]][1]
        scale = torch.stack([_row_scales(W[n:n + _GROUP], largest).amax(0) for n in range(0, W.shape[0], _GROUP)])
        of_row, of_column = (torch.arange(n, device="cuda") // _GROUP for n in W.shape)
        return W / scale[of_row[:, None], of_column] if case["w"] == "e4m3" else None, scale
    if op == "quant":
        y, H = st["X"].double(), None
    else:
        h = st["X"].double() + (0.0 if st["residual"] is None else st["residual"].double())
        y = h / ((h * h).sum(1, keepdim=True) / h.shape[1] + st["eps"]).sqrt() * st["gamma"].double()
        H = None if st["residual"] is None else h
        if case["out"] == "bf16":
            return y, H
    scale = _row_scales(y, _FORMATS[case["out"]][1])
    codes = y / scale[:, torch.arange(y.shape[1], device="cuda") // _GROUP] if case["out"] == "e4m3" else None
    return (codes, scale) if op == "quant" else (codes, scale, H)


def work(case):
    op = case["op"]
    if op == "linear":
        d_in, d_out, b = case["d_in"], case["d_out"], case["b"]
        groups = math.ceil(d_in / _GROUP)
        return {"bytes": b * d_in + d_out * d_in + 4 * groups * (b + math.ceil(d_out / _GROUP)) + 2 * b * d_out, "flops": 2 * b * d_in * d_out}
    if op == "pack":
        d_in, d_out = case["d_in"], case["d_out"]
        return {"bytes": (3 if case["from"] == "bf16" else 5) * d_in * d_out + 4 * math.ceil(d_in / _GROUP) * math.ceil(d_out / _GROUP),
                "flops": 2 * d_in * d_out}
    b, d = case["b"], case["d"]
    out = 2 * b * d if case["out"] == "bf16" else b * d + 4 * b * math.ceil(d / _GROUP)
    if op == "quant":
        return {"bytes": 2 * b * d + out, "flops": 2 * b * d}
    return {"bytes": 2 * b * d + 2 * d + (4 * b * d if case["residual"] else 0) + out, "flops": 6 * b * d}
