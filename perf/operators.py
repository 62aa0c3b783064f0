"""The operators before the hot path, at the sizes a training program calls them: a layer's
activations packed to 8 bits, and what its forward and backward pass computes from them.

Five operators ("op" of a case):
  pack     a matrix to 8-bit floating point (e4m3) with a power-of-two scale for every block of
           128: along the rows for activations (gtopk_pack_rows), or for tiles of 128 x 128 with
           the transposed matrix beside it for weights (gtopk_pack_tiles)
  unpack   a packed checkpoint back to values, through the layer's activation (gtopk_unpack)
  actgrad  dx = dy * f'(x) with x from a packed checkpoint (gtopk_activation_grad)
  product  C = A B^T of two packed matrices: a layer's forward product, or its input gradient
           (gtopk_scaled_product)
  wgrad    every worker's weight gradient dY^T X with X from a packed checkpoint, written into
           the workers' gradient rows (gtopk_weight_grad)

Layer sizes are those of the fully connected layers of this repository's AlexNet workload
(9216 -> 4096 -> 4096 -> 1000), at up to 32 workers with some tens of samples each, and generic
ones.
"""
import math
import random

import torch

own = False

BLOCK = 128
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _ceil(a, b):
    return -(-a // b)


def listed():
    return [
        # the inputs of the first fully connected layer, 32 workers with 64 samples each, to a checkpoint
        {"name": "pack_input", "op": "pack", "tiles": False, "rows": 2048, "cols": 9216, "dtype": "bf16"},
        # the master weights of that layer after an update, for the next iteration's two products
        {"name": "pack_weights", "op": "pack", "tiles": True, "rows": 4096, "cols": 9216, "dtype": "f32"},
        # the next layer's input recomputed from one sample's checkpoint: latency
        {"name": "unpack_one", "op": "unpack", "act": "relu", "rows": 1, "cols": 4096, "dtype": "bf16"},
        # a hidden layer's input recomputed for a long batch
        {"name": "unpack_gelu", "op": "unpack", "act": "gelu", "rows": 8192, "cols": 4096, "dtype": "bf16"},
        # the backward of a hidden layer's activation, 32 workers
        {"name": "actgrad_relu", "op": "actgrad", "act": "relu", "rows": 8192, "cols": 4096, "dtype": "bf16"},
        # a small layer of odd width, in 32 bits
        {"name": "actgrad_odd", "op": "actgrad", "act": "tanh", "rows": 777, "cols": 1001, "dtype": "f32"},
        # one sample through the first fully connected layer: the weights are read once
        {"name": "product_one", "op": "product", "M": 1, "N": 4096, "K": 9216, "dtype": "bf16"},
        # the forward product of that layer, 32 workers with 64 samples each
        {"name": "product_forward", "op": "product", "M": 2048, "N": 4096, "K": 9216, "dtype": "bf16"},
        # the input gradient of the same layer for a large batch, its last samples missing: the largest product
        {"name": "product_input_grad", "op": "product", "M": 8187, "N": 9216, "K": 4096, "dtype": "f32"},
        # the weight gradients of the first fully connected layer into the rows of 16 workers
        {"name": "wgrad_workers", "op": "wgrad", "P": 16, "rows": 1024, "N": 4096, "K": 9216, "dtype": "bf16",
         "ragged": False, "behind": 1001},
        # the last layer (1000 classes) in 32 bits, the samples spread unevenly over the workers, at an odd place of the rows
        {"name": "wgrad_ragged", "op": "wgrad", "P": 8, "rows": 1501, "N": 1000, "K": 4096, "dtype": "f32",
         "ragged": True, "behind": 1001},
        # a long batch of one worker, a square layer: one product over the whole batch
        {"name": "wgrad_long", "op": "wgrad", "P": 1, "rows": 16384, "N": 1024, "K": 1024, "dtype": "bf16",
         "ragged": False, "behind": 0},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["pack", "unpack", "actgrad", "product", "product", "wgrad", "wgrad"])
    if op == "pack":
        tiles = rng.random() < 0.4
        return {"op": op, "tiles": tiles, "rows": _log(rng, 1, 8192), "cols": _log(rng, 8, 9216),
                "dtype": "f32" if tiles else rng.choice(["bf16", "bf16", "f16", "f32"])}
    if op in ("unpack", "actgrad"):
        return {"op": op, "act": rng.choice(["none", "relu", "tanh", "sigmoid", "silu", "gelu"]),
                "rows": _log(rng, 1, 8192), "cols": _log(rng, 8, 9216), "dtype": rng.choice(["bf16", "bf16", "f16", "f32"])}
    if op == "product":
        return {"op": op, "M": _log(rng, 1, 8192), "N": _log(rng, 16, 6144), "K": _log(rng, 64, 6144),
                "dtype": rng.choice(["bf16", "bf16", "f16", "f32"])}
    P = 2 ** rng.randint(0, 5)
    return {"op": op, "P": P, "rows": P * _log(rng, 1, 16384 // P), "N": _log(rng, 8, 2048), "K": _log(rng, 8, 2048),
            "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "ragged": rng.random() < 0.5, "behind": rng.choice([0, 0, 7, 1001])}


# ---- inputs -------------------------------------------------------------------------

def _activations(rows, cols, gen):
    """Values as they come out of a layer: features of very different scale, some of them outliers."""
    scale = torch.exp(torch.randn(cols, device="cuda", generator=gen))
    scale = torch.where(torch.rand(cols, device="cuda", generator=gen) < 0.005, scale * 20.0, scale)
    return torch.randn(rows, cols, device="cuda", generator=gen) * scale


def _weights(rows, cols, gen):
    return torch.randn(rows, cols, device="cuda", generator=gen) * (1.0 / math.sqrt(cols))


def _output_gradient(rows, cols, gen):
    """Small, with samples of very different weight, and a last row of padding (all zero)."""
    d = torch.randn(rows, cols, device="cuda", generator=gen) * 1e-3
    d = d * torch.exp(torch.randn(rows, 1, device="cuda", generator=gen))
    if rows > 1:
        d[-1] = 0.0
    return d


def _packed(x, tiles=False):
    """The plain form's packed matrix, with rows as long as the library wants them: whole blocks of codes, scales in fours."""
    rows, cols = x.shape
    codes, exps = _pack_plain(x, tiles)
    c = torch.zeros(rows, _ceil(cols, BLOCK) * BLOCK, dtype=torch.uint8, device="cuda")
    c[:, :cols] = codes.view(torch.uint8)
    s = torch.zeros(rows, _ceil(exps.shape[1], 4) * 4, dtype=torch.uint8, device="cuda")
    s[:, :exps.shape[1]] = exps
    return c, s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1_000_003 * int(seed) + 17)
    s = dict(case)
    u8 = dict(dtype=torch.uint8, device="cuda")
    if case["op"] == "wgrad":
        P, R, N, K = case["P"], case["rows"], case["N"], case["K"]
        s["codes"], s["scales"] = _packed(_activations(R, K, gen).relu_())
        s["dy"] = _output_gradient(R, N, gen).to(TYPES[case["dtype"]])
        # the plan of the batch, which the program has on the host: the samples of each worker
        length, r = [R // P] * P, random.Random("%d %d" % (int(seed), R))
        if case["ragged"] and P > 1:     # uneven shares, one worker with none
            cuts = sorted(r.randint(0, R) for _ in range(P - 1))
            length = [b - a for a, b in zip([0] + cuts, cuts + [R])]
            length[1] += length[0]
            length[0] = 0
        begin = [0]
        for n in length:
            begin.append(begin[-1] + n)
        s["longest"] = max(length)
        s["begin"] = torch.tensor(begin, dtype=torch.int32, device="cuda")
        # the workers' gradient rows: this layer's part lies behind `behind` elements of other layers
        s["grad"] = torch.zeros(P, case["behind"] + N * K, device="cuda")
        return s
    if case["op"] == "product":
        M, N, K = case["M"], case["N"], case["K"]
        s["a"] = _packed(_activations(M, K, gen))
        s["b"] = _packed(_weights(N, K, gen), tiles=True)
        s["out"] = torch.empty(M, N, dtype=TYPES[case["dtype"]], device="cuda")
        return s
    rows, cols, t = case["rows"], case["cols"], TYPES[case["dtype"]]
    if case["op"] == "pack":
        s["x"] = (_weights if case["tiles"] else _activations)(rows, cols, gen).to(t)
        s["codes"] = torch.empty(rows, _ceil(cols, BLOCK) * BLOCK, **u8)
        s["scales"] = torch.empty(rows, _ceil(_ceil(cols, BLOCK), 4) * 4, **u8)
        if case["tiles"]:
            s["codes_t"] = torch.empty(cols, _ceil(rows, BLOCK) * BLOCK, **u8)
            s["scales_t"] = torch.empty(cols, _ceil(_ceil(rows, BLOCK), 4) * 4, **u8)
        return s
    s["codes"], s["scales"] = _packed(_activations(rows, cols, gen))
    s["out"] = torch.empty(rows, cols, dtype=t, device="cuda")
    if case["op"] == "actgrad":
        s["dy"] = _output_gradient(rows, cols, gen).to(t)
    return s


# ---- the plain forms ----------------------------------------------------------------

def _pow2(e):
    """2^e as float32 for e in -126 .. 127."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _pack_plain(x, tiles=False):
    """(codes as float8, exponents + 127): the smallest power of two that brings a block's largest magnitude to 448 or less."""
    rows, cols = x.shape
    nb, nr = _ceil(cols, BLOCK), _ceil(rows, BLOCK)
    y = x.float()
    p = torch.nn.functional.pad(y.abs(), (0, nb * BLOCK - cols, 0, nr * BLOCK - rows if tiles else 0))
    amax = p.view(nr, BLOCK, nb, BLOCK).amax(dim=(1, 3)) if tiles else p.view(rows, nb, BLOCK).amax(dim=2)
    m, q = torch.frexp(amax)
    e = torch.where(m <= 0.875, q - 9, q - 8).to(torch.int32)
    e = torch.where(amax == 0, -127, e).clamp(min=-127)
    if tiles:
        e = e.repeat_interleave(BLOCK, dim=0)[:rows]
    per_value = _pow2(-e).repeat_interleave(BLOCK, dim=1)[:, :cols]
    return (y * per_value).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _values(codes, scales, cols):
    """The values of a packed matrix, in 32 bits."""
    nb = _ceil(cols, BLOCK)
    s = scales[:, :nb].to(torch.int32)
    f = torch.where(s == 0, 0x00400000, s << 23).view(torch.float32)
    return codes[:, :cols].contiguous().view(torch.float8_e4m3fn).float() * f.repeat_interleave(BLOCK, dim=1)[:, :cols]


def _act(name, x):
    if name == "relu":
        return x.clamp(min=0)
    if name == "tanh":
        return torch.tanh(x)
    if name == "sigmoid":
        return torch.sigmoid(x)
    if name == "silu":
        return x * torch.sigmoid(x)
    if name == "gelu":
        return x * 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5)))
    return x


def _act_slope(name, x):
    if name == "relu":
        return (x > 0).to(x.dtype)
    if name == "tanh":
        t = torch.tanh(x)
        return (1.0 - t) * (1.0 + t)
    if name == "sigmoid":
        return torch.sigmoid(x) * torch.sigmoid(-x)
    if name == "silu":
        g = torch.sigmoid(x)
        return g * (1.0 + x * torch.sigmoid(-x))
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))
    return torch.ones_like(x)


def _rows_of_workers(s, x):
    """x[rows] as [P][longest]: every worker's rows, zero behind its last one."""
    if not s["ragged"]:
        return x.reshape(s["P"], s["rows"] // s["P"], -1)
    at = s["begin"][:-1, None] + torch.arange(max(1, s["longest"]), device=x.device)
    inside = at < s["begin"][1:, None]
    return torch.where(inside[:, :, None], x[at.clamp(max=s["rows"] - 1)], 0)


def run(state):
    s = state
    if own:
        return _run_own(s)
    op = s["op"]
    if op == "pack":
        codes, exps = _pack_plain(s["x"], s["tiles"])
        out = {"codes": codes, "scales": exps.view(torch.float8_e8m0fnu)}
        if s["tiles"]:
            codes, exps = _pack_plain(s["x"].t().contiguous(), True)
            out.update(codes_t=codes, scales_t=exps.view(torch.float8_e8m0fnu))
        return out
    if op == "unpack":
        return _act(s["act"], _values(s["codes"], s["scales"], s["cols"])).to(s["out"].dtype)
    if op == "actgrad":
        return (s["dy"].float() * _act_slope(s["act"], _values(s["codes"], s["scales"], s["cols"]))).to(s["out"].dtype)
    if op == "product":
        return (_values(*s["a"], s["K"]) @ _values(*s["b"], s["K"]).t()).to(s["out"].dtype)
    d = _rows_of_workers(s, s["dy"].float())
    x = _rows_of_workers(s, _values(s["codes"], s["scales"], s["K"]))
    return torch.bmm(d.transpose(1, 2).contiguous(), x)


def _run_own(s):
    from paper_1901_04359_amd import binding as B
    op = s["op"]
    if op == "pack":
        rows, cols = s["rows"], s["cols"]
        if s["tiles"]:
            B.gtopk_pack_tiles(s["x"], s["codes"], s["scales"], s["codes_t"], s["scales_t"])
        else:
            B.gtopk_pack_rows(s["x"], s["codes"], s["scales"])
        e4m3, e8m0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
        out = {"codes": s["codes"].view(e4m3)[:, :cols], "scales": s["scales"].view(e8m0)[:, :_ceil(cols, BLOCK)]}
        if s["tiles"]:
            out.update(codes_t=s["codes_t"].view(e4m3)[:, :rows], scales_t=s["scales_t"].view(e8m0)[:, :_ceil(rows, BLOCK)])
        return out
    if op == "unpack":
        B.gtopk_unpack(s["codes"], s["scales"], s["act"], s["out"])
        return s["out"]
    if op == "actgrad":
        B.gtopk_activation_grad(s["codes"], s["scales"], s["act"], s["dy"], s["out"])
        return s["out"]
    if op == "product":
        M, N, K = s["M"], s["N"], s["K"]
        if "ws" not in s:                # kept by the program, as every workspace of the library
            s["ws"] = B.alloc_product_workspace(M, N, K)
        B.gtopk_scaled_product(*s["a"], *s["b"], K, s["out"], s["ws"])
        return s["out"]
    P, N, K = s["P"], s["N"], s["K"]
    if "ws" not in s:
        s["ws"] = B.alloc_weight_grad_workspace(s["rows"], P, N, K)
    grad = s["grad"][:, s["behind"]:].unflatten(1, (N, K))
    B.gtopk_weight_grad(s["dy"], s["codes"], s["scales"], s["begin"] if s["ragged"] else None, grad, False, s["ws"])
    return grad


def work(case):
    op = case["op"]
    if op == "wgrad":
        P, R, N, K = case["P"], case["rows"], case["N"], case["K"]
        return {"bytes": R * N * BYTES[case["dtype"]] + R * K + R * _ceil(K, BLOCK) + 4 * P * N * K, "flops": 2 * R * N * K}
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": (M + N) * (K + _ceil(K, BLOCK)) + M * N * BYTES[case["dtype"]], "flops": 2 * M * N * K}
    rows, cols, b = case["rows"], case["cols"], BYTES[case["dtype"]]
    packed = rows * (cols + _ceil(cols, BLOCK))
    if op == "pack":
        return {"bytes": rows * cols * b + packed + (cols * (rows + _ceil(rows, BLOCK)) if case["tiles"] else 0), "flops": 0}
    return {"bytes": packed + rows * cols * b * (2 if op == "actgrad" else 1), "flops": 0}


# ---- the operators' definitions in 64 bits ------------------------------------------

def _decoded(codes, scales, cols):
    """Sign, four exponent bits (bias 7, 0: subnormal), three mantissa bits; times 2^(scale - 127)."""
    c = codes[:, :cols].to(torch.int64)
    exponent, mantissa = (c >> 3) & 15, (c & 7).double()
    v = torch.where(exponent == 0, mantissa * 2.0 ** -9, (8.0 + mantissa) * torch.exp2((exponent - 10).double()))
    v = torch.where(c >= 128, -v, v)
    block = torch.div(torch.arange(cols, device=codes.device), BLOCK, rounding_mode="floor")
    return v * torch.exp2(scales[:, block].double() - 127.0)


def _nearest(t):
    """The nearest number of four significant bits with an exponent of at least -6, ties to the even one."""
    e = torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -60))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return torch.round(t / step) * step


def _pack_exact(x, by_rows):
    x = x.double()
    codes, scales = torch.empty_like(x), []
    for j in range(0, x.shape[1], BLOCK):
        b = x[:, j:j + BLOCK]
        top = b.abs().amax(dim=1, keepdim=True)
        if not by_rows:
            top = torch.cat([t.amax(dim=0, keepdim=True).expand(t.shape[0], 1) for t in top.split(BLOCK)])
        e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0)).clamp(min=-127)
        e = torch.where(top > 448.0 * torch.exp2(e), e + 1, e)           # the logarithm's rounding, either way
        e = torch.where((top <= 448.0 * torch.exp2(e - 1)) & (e > -127), e - 1, e)
        codes[:, j:j + BLOCK] = _nearest(b / torch.exp2(e))
        scales.append(torch.exp2(e))
    return codes, torch.cat(scales, dim=1)


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == "pack":
        codes, scales = _pack_exact(s["x"], not s["tiles"])
        out = {"codes": codes, "scales": scales}
        if s["tiles"]:
            codes, scales = _pack_exact(s["x"].t(), False)
            out.update(codes_t=codes, scales_t=scales)
        return out
    if op == "product":
        return _decoded(*s["a"], s["K"]) @ _decoded(*s["b"], s["K"]).t()
    if op == "wgrad":
        x, d, at = _decoded(s["codes"], s["scales"], s["K"]), s["dy"].double(), s["begin"].tolist()
        out = torch.empty(s["P"], s["N"], s["K"], dtype=torch.float64, device="cuda")
        for w in range(s["P"]):
            out[w] = d[at[w]:at[w + 1]].t() @ x[at[w]:at[w + 1]]
        return out
    x = _decoded(s["codes"], s["scales"], s["cols"])
    up, down = torch.exp(-x.clamp(min=-700)), torch.exp(x.clamp(max=700))
    g = 1.0 / (1.0 + up)                                                 # the logistic function
    h = 0.5 * torch.special.erfc(-x / math.sqrt(2.0))                    # the normal distribution function
    f = s["act"]
    if op == "unpack":
        return {"none": x, "relu": torch.where(x > 0, x, 0.0), "tanh": torch.tanh(x), "sigmoid": g, "silu": x * g, "gelu": x * h}[f]
    density = torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    slope = {"none": torch.ones_like(x), "relu": torch.where(x > 0, 1.0, 0.0), "tanh": 1.0 / torch.cosh(x.clamp(-300, 300)) ** 2,
             "sigmoid": g / (1.0 + down), "silu": g + x * g / (1.0 + down), "gelu": h + x * density}[f]
    return s["dy"].double() * slope
