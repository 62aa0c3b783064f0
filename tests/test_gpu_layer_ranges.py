"""The layer calls at the ends of their ranges: values that fp32 cannot hold, the tails of the activation functions, scales from
the smallest on, and the sizes at which a weight gradient takes its large tiles or bands of tiles.

Tolerances are derived beside the tests.  u = 2^-24 is half a step of fp32."""
import math

import numpy as np
import pytest

from tests import layer_reference as ref
from tests.gpu_harness import say
from tests.test_gpu_layer import TYPES, half_step, packed_on_gpu, torch_type, values_in

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "tanh", "sigmoid", "silu", "gelu"]


# ---- values that fp32 cannot hold -----------------------------------------------------

@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_activation_of_values_that_fp32_cannot_hold(act, dtype):
    """All codes but NaN's at the largest scales: f(x) and f'(x) are x, 0, 1 or -1 there (from |x| = 2^110 on; at 0 also
    1/2), and a value of 2^128 or more gives what it tends to, an infinity only where f is unbounded."""
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    magnitudes = np.arange(0x7F, dtype=np.uint8)
    codes = np.zeros((4, 256), np.uint8)
    codes[:, :127], codes[:, 128:255] = magnitudes, magnitudes | 0x80
    scales = np.repeat(np.array([[246], [247], [250], [254]], np.uint8), 2, axis=1)
    x = ref.values(codes, scales, 256)
    c, s = packed_on_gpu(codes, scales)
    out, dx = torch.zeros(4, 256, dtype=t, device="cuda"), torch.zeros(4, 256, dtype=t, device="cuda")
    dy = torch.tensor([1.0, -0.5, 3.0, 0.0], dtype=t, device="cuda")[:, None].expand(4, 256).contiguous()
    say(f"layer: {act} {dtype} of values that fp32 cannot hold")
    B.gtopk_unpack(c, s, act, out)
    B.gtopk_activation_grad(c, s, act, dy, dx)
    for got, want in ((out, ref.act(act, x)), (dx, dy.double().cpu().numpy() * ref.slope(act, x))):
        want = torch.from_numpy(want).float().to(t).double()
        got = got.double().cpu()
        assert not bool(torch.isnan(got).any()), act
        assert torch.equal(torch.isinf(got), torch.isinf(want)), act
        fine = ~torch.isinf(want)
        # (32 u for the functions, at 1/2 and 1; a step of the type where that moves a value over a rounding border)
        assert bool(((got - want).abs()[fine] <= (32 * 2.0 ** -24 + 2 * half_step(t)) * want.abs()[fine]).all()), act


# ---- the tails of the activation functions --------------------------------------------

@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_activation_relative_to_its_value(act, dtype):
    """Every code at scales that lead from 2^-69 far behind the last argument at which an exponential is not 0: errors relative to f and f'.

    In fp32 an exponential of a corrected argument is off by 4 u (1 step of 2 u of the instruction, the correction's rounding and
    the last fma), a reciprocal by 2 u, a sum or product by 1 u.  With e = exp(-|x|) (tanh: exp(-2 |x|)), whose error
    enters with the factor in brackets:
      logistic  1 / (1 + e): 4 (1/2) + 1 + 2 = 5;  e / (1 + e): 4 (1) + 1 + 2 + 1 = 8;  SiLU 1 more
      tanh      (1 - e) / (1 + e), |x| >= 1/4: 4 (2 e / (1 - e^2) <= 1.93) + 1 + 1 + 2 + 1 = 13; below a series to x^9, which leaves out
                1382/155925 x^10 < 0.2 u, and some roundings
      slopes    4 e / (1 + e)^2 and e / (1 + e)^2: 4 (1) + 2 (1 + 2) + 3 = 13; SiLU's is the sum of two such terms, and is held against
                the sum of their magnitudes, as is GELU's
      GELU      |x| bell tail: 4 for the bell, 3 roundings, and the tail's polynomial with its reciprocal 14.4 (all arguments in steps of 3e-5,
                emulated with the reciprocal a step off to either side): 22
    Below: 16 u, GELU 24 u.  For 16 bits the exponentials' arguments are not corrected: up to |x| u more, in GELU x^2 u.  An
    exponential below 2^-126 may be 0."""
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    codes = np.tile(np.concatenate([np.arange(0x7F), [0], np.arange(0x80, 0xFF), [0]]).astype(np.uint8), (75, 1))
    scales = np.repeat(np.arange(67, 142, dtype=np.uint8)[:, None], 2, axis=1)
    scales[0] = 60
    x = ref.values(codes, scales, 256)
    x[x == 0] = 0.0
    c, s = packed_on_gpu(codes, scales)
    out, dx = torch.zeros(75, 256, dtype=t, device="cuda"), torch.zeros(75, 256, dtype=t, device="cuda")
    say(f"layer: {act} {dtype} relative to its value")
    B.gtopk_unpack(c, s, act, out)
    B.gtopk_activation_grad(c, s, act, torch.ones(75, 256, dtype=t, device="cuda"), dx)
    f, slope = ref.act(act, x), ref.slope(act, x)
    size = np.abs(slope)
    logistic = ref.act("sigmoid", x)
    if act == "silu":
        size = logistic + np.abs(x) * logistic * ref.act("sigmoid", -x)
    if act == "gelu":
        size = np.abs(ref.act("gelu", x) / np.where(x == 0, 1.0, x)) + np.abs(x) * np.exp(-x * x / 2) / math.sqrt(2 * math.pi)
        size[x == 0] = 0.5
    u, floor = 2.0 ** -24, 2.0 ** -126 * np.maximum(1.0, np.abs(x))
    rel = (0.0 if act in ("none", "relu") else 24 * u if act == "gelu" else 16 * u) + np.zeros_like(x)
    if dtype != "f32":
        rel = rel + u * (np.minimum(np.abs(x), 128) + np.minimum(x * x, 256)) + half_step(t)
        floor = floor + (2.0 ** -25 if dtype == "f16" else 0.0)
    for got, want, of in ((out, f, np.abs(f)), (dx, slope, size)):
        g = got.double().cpu().numpy()
        fits = np.abs(want) < torch.finfo(t).max              # (fp16 ends at 65504)
        assert np.isinf(g[~fits]).all()
        off = np.abs(g - want) - floor
        bad = fits & (off > rel * of)
        assert not bad.any(), (act, x[bad][:5], g[bad][:5], want[bad][:5])


# ---- products and weight gradients of every scale -------------------------------------

def int_codes(rows, cols, seed, unit=1.0):
    """Codes of -2, -1, 0, 1 and 2 times `unit` (a power of two), padded with zeros to whole blocks."""
    r = np.random.default_rng([rows, cols, seed, 17])
    codes = np.zeros((rows, -(-cols // 128) * 128), np.uint8)
    codes[:, :cols] = ref.encode(r.integers(-2, 3, (rows, cols)) * unit)
    return codes


# (all of a product's kernels: 16 and 32 rows without tiles, tiles of 128 in one piece and in shares of K, tiles of 256)
@pytest.mark.parametrize("M,N,K", [(3, 40, 700), (20, 33, 1500), (130, 140, 300), (70, 150, 2500), (2817, 2850, 700)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("unit", [1.0, 64.0, 2.0 ** -6])
def test_product_of_every_scale_that_pack_makes(M, N, K, dtype, unit):
    """A's scales 0 to 247 and B's, block by block, as far from them as brings the products near 1 (2^-7 at the least).  Every value is
    a multiple of 2^-133, and a sum one of fewer than 2^23 units of 2^-7 unit^2: exact in every type's path."""
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    nb = -(-K // 128)
    r = np.random.default_rng([M, N, K])
    each = r.permutation(np.concatenate([[0, 247], r.integers(0, 248, nb)])[:nb])
    a, b = int_codes(M, K, 1, unit), int_codes(N, K, 2, 1.0)
    sa, sb = np.tile(each.astype(np.uint8), (M, 1)), np.tile(np.clip(254 - each, 7, 247).astype(np.uint8), (N, 1))
    want = torch.from_numpy(ref.values(a, sa, K) @ ref.values(b, sb, K).T)
    assert float(want.abs().max()) * 2.0 ** 7 / unit < 2 ** 24
    out = torch.zeros(M, N, dtype=t, device="cuda")
    ws = B.alloc_product_workspace(M, N, K)
    say(f"layer: product {M}x{N}x{K} {dtype} unit {unit}, scales from 0")
    B.gtopk_scaled_product(*packed_on_gpu(a, sa), *packed_on_gpu(b, sb), K, out, ws)
    assert torch.equal(out.cpu(), want.float().to(t))
    turned = torch.zeros(N, M, dtype=t, device="cuda")
    B.gtopk_scaled_product(*packed_on_gpu(b, sb), *packed_on_gpu(a, sa), K, turned, B.alloc_product_workspace(N, M, K))
    assert torch.equal(turned.cpu(), want.T.float().to(t))


@pytest.mark.parametrize("M,N,K", [(3, 40, 300), (20, 33, 3000), (70, 150, 2500), (200, 4097, 1030), (2817, 2850, 300)])
def test_product_of_values_that_fp32_cannot_hold(M, N, K):
    """In rows 1 and 2 of A stand 2^128 and -2^128, with products of 2^108 and -2^108, and in B's last row a NaN: values count as
    they are, in every type that can hold the result."""
    import torch
    from paper_1901_04359_amd import binding as B
    a, b = int_codes(M, K, 3), np.abs(int_codes(N, K, 4))
    nb = -(-K // 128)
    b[:, :K] = 0x38                          # ones
    sa, sb = np.full((M, nb), 127, np.uint8), np.full((N, nb), 107, np.uint8)
    a[1, :], sa[1, :] = 0, 247
    a[1, 5] = 0x78                           # 256 * 2^120
    a[2, :], sa[2, :] = 0, 247
    a[2, K - 1] = 0xF8
    b[N - 1, K - 2] = 0x7F
    b[N - 2, (nb - 1) * 128:], sb[N - 2, nb - 1] = 0, 254     # zeros at the largest scale
    want = torch.from_numpy(ref.values(a, sa, K) @ ref.values(b, sb, K).T)
    assert bool((want[1, :N - 2] == 2.0 ** 108).all()) and bool((want[2, :N - 2] == -2.0 ** 108).all())
    say(f"layer: product {M}x{N}x{K} of 2^128")
    for dtype in TYPES:
        t = torch_type(dtype)
        out = torch.zeros(M, N, dtype=t, device="cuda")
        B.gtopk_scaled_product(*packed_on_gpu(a, sa), *packed_on_gpu(b, sb), K, out, B.alloc_product_workspace(M, N, K))
        w, got = want.float().to(t), out.cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(w)) and int(torch.isnan(w).sum()) == M
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(w))


@pytest.mark.parametrize("M,N,K", [(3, 40, 300), (20, 40, 300), (130, 140, 300), (2817, 2850, 300)])
def test_product_of_values_below_the_normal_range(M, N, K):
    """All codes of A at scales 0 to 9, B's values powers of two that bring them near 1.  To fp32 a value of A below 2^-126 may
    be rounded to a multiple of 2^-133: half of one, 2^-134, off."""
    import torch
    from paper_1901_04359_amd import binding as B
    r = np.random.default_rng([M, N, K, 5])
    nb = -(-K // 128)
    a, b = np.zeros((M, nb * 128), np.uint8), np.zeros((N, nb * 128), np.uint8)
    a[:, :K] = r.integers(0, 127, (M, K)) | r.integers(0, 2, (M, K)) * 128
    b[:, :K] = ref.encode(np.exp2(r.integers(-3, 4, (N, K)).astype(np.float64)))
    sa, sb = r.integers(0, 10, (M, nb)).astype(np.uint8), np.full((N, nb), 247, np.uint8)
    va, vb = ref.values(a, sa, K), ref.values(b, sb, K)
    want, size = va @ vb.T, np.abs(va) @ np.abs(vb).T
    lost = 2.0 ** -134 * ((np.abs(va) < 2.0 ** -126) * 1.0 @ np.abs(vb).T)
    say(f"layer: product {M}x{N}x{K} of values below the normal range")
    out = torch.zeros(M, N, device="cuda")
    B.gtopk_scaled_product(*packed_on_gpu(a, sa), *packed_on_gpu(b, sb), K, out, B.alloc_product_workspace(M, N, K))
    assert (np.abs(out.double().cpu().numpy() - want) <= (K + 4) * 2.0 ** -23 * size + lost).all()


def power_rows(rows, N, scales, seed):
    """dY of -2, .. 2 times 2^(127 - the row's scale), so that products with X in that scale are small integers."""
    r = np.random.default_rng([rows, N, seed, 23])
    return r.integers(-2, 3, (rows, N)) * np.exp2(127.0 - scales.astype(np.float64))[:, None]


# (tiles of 128 and of 128 x 256, in one piece and in shares of the rows; the other kernels: test_gpu_layer_plans.py)
@pytest.mark.parametrize("P,rows,N,K", [(2, 60, 33, 200), (2, 60, 40, 640), (1, 3000, 40, 300), (1, 2000, 1030, 1030), (3, 900, 130, 700)])
@pytest.mark.parametrize("dtype,low,high", [("f32", 1, 247), ("bf16", 1, 247), ("f16", 114, 140)])
@pytest.mark.parametrize("unit", [1.0, 64.0])
def test_weight_grad_of_every_scale(P, rows, N, K, dtype, low, high, unit):
    """X's scales over their whole range, as far as dY's type can make up for them (2 * 2^126 at scale 1): every product is an
    integer times unit of at most 4, every sum exact, and what X decodes to a multiple of 2^-133."""
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    r = np.random.default_rng([P, rows, N, K, high])
    per_row = r.integers(low, high + 1, rows).astype(np.uint8)
    per_row[:2] = low, high
    codes, scales = int_codes(rows, K, 7, unit), np.repeat(per_row[:, None], -(-K // 128), axis=1)
    dy = power_rows(rows, N, per_row, 8)
    d = torch.from_numpy(dy).to(t)
    assert np.array_equal(d.double().numpy(), dy)
    want = torch.from_numpy(ref.weight_grad(dy, ref.values(codes, scales, K), [rows // P * w for w in range(P + 1)])).float()
    grad = torch.empty(P, N, K, device="cuda")
    say(f"layer: weight_grad {dtype} P {P} rows {rows} {N}x{K} unit {unit}, scales {low} to {high}")
    B.gtopk_weight_grad(d.cuda(), *packed_on_gpu(codes, scales), None, grad, False, B.alloc_weight_grad_workspace(rows, P, N, K))
    assert torch.equal(grad.cpu(), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("P,rows,N,K", [(2, 60, 33, 200), (2, 60, 40, 640), (1, 2000, 1030, 1030)])
def test_weight_grad_of_values_at_both_ends(dtype, P, rows, N, K):
    """Below 2^-126 a value of X may be rounded to a multiple of 2^-133, half of one off; one of 2^128 or more, or a NaN scale, makes
    the sums it enters infinite or NaN, in its column of its worker's gradient and nowhere else."""
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    r = np.random.default_rng([P, rows, N, K, 6])
    nb, each = -(-K // 128), rows // P
    begin = [each * w for w in range(P + 1)]
    codes = np.zeros((rows, nb * 128), np.uint8)
    codes[:, :K] = r.integers(0, 127, (rows, K)) | r.integers(0, 2, (rows, K)) * 128
    scales = r.integers(0, 10, (rows, nb)).astype(np.uint8)
    dy = np.exp2(r.integers(10, 15, (rows, N)).astype(np.float64)) * r.choice([-1.0, 1.0], (rows, N))
    x = ref.values(codes, scales, K)
    want, size = ref.weight_grad(dy, x, begin), ref.weight_grad(np.abs(dy), np.abs(x), begin)
    lost = 2.0 ** -134 * ref.weight_grad(np.abs(dy), (np.abs(x) < 2.0 ** -126) * 1.0, begin)
    grad = torch.empty(P, N, K, device="cuda")
    ws = B.alloc_weight_grad_workspace(rows, P, N, K)
    say(f"layer: weight_grad {dtype} P {P} rows {rows} {N}x{K} of values below the normal range")
    B.gtopk_weight_grad(torch.from_numpy(dy).to(t).cuda(), *packed_on_gpu(codes, scales), None, grad, False, ws)
    # (a sum that passes below 2^-126 may lose what is below it, once per addition)
    assert (np.abs(grad.double().cpu().numpy() - want) <= (each + 4) * (2.0 ** -23 * size + 2.0 ** -126) + lost).all()

    codes = int_codes(rows, K, 9)
    codes[codes == 0] = 0x38
    codes[:, K:] = 0
    scales = np.full((rows, nb), 127, np.uint8)
    codes[3, 1], scales[3, 0] = 0x78, 247                     # 2^128; the row's other values of the block are 2^120 and 2^121
    codes[4, 2], scales[4, 0] = 0xFE, 254
    scales[5, nb - 1] = 255
    dy = np.ones((rows, N))
    say(f"layer: weight_grad {dtype} P {P} rows {rows} {N}x{K} of 2^128 and NaN")
    B.gtopk_weight_grad(torch.from_numpy(dy).to(t).cuda(), *packed_on_gpu(codes, scales), None, grad, False, ws)
    x = ref.values(codes, scales, K)
    far = np.stack([~(np.abs(x[a:b]) < 2.0 ** 128).all(axis=0) for a, b in zip(begin[:-1], begin[1:])])       # [P][K]
    assert far[0].sum() >= 2 and not far[1:].any()
    got = grad.cpu().double().numpy()
    fine = np.isfinite(got)
    assert np.array_equal(fine, np.repeat(~far[:, None, :], N, axis=1))
    want, size = ref.weight_grad(dy, np.where(np.repeat(far, each, axis=0), 0.0, x), begin), ref.weight_grad(dy, np.abs(x), begin)
    assert (np.abs(got - want)[fine] <= ((each + 4) * 2.0 ** -23 * size)[fine]).all()

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K", [(1, 300, 5000), (16, 130, 1000), (17, 90, 2050), (32, 300, 4096)])
def test_product_of_few_rows_holds_fp32_sums(M, N, K, dtype):
    """Reading B bounds these, whatever the products: a 16-bit result is the fp32 sum, off by at most (K + 4) 2^-23 of the magnitudes, rounded
    once, also where the sum cancels."""
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    a, b = ref.pack(values_in(M, K, 41)), ref.pack(values_in(N, K, 42) / math.sqrt(K), tiles=True)
    va, vb = ref.values(*a, K), ref.values(*b, K)
    out = torch.zeros(M, N, dtype=t, device="cuda")
    say(f"layer: product {M}x{N}x{K} to {dtype}, fp32 sums")
    B.gtopk_scaled_product(*packed_on_gpu(*a), *packed_on_gpu(*b), K, out, B.alloc_product_workspace(M, N, K))
    want, bound = va @ vb.T, (K + 4) * 2.0 ** -23 * (np.abs(va) @ np.abs(vb).T)
    err = np.abs(out.double().cpu().numpy() - want)
    assert (err <= bound * (1 + half_step(t)) + half_step(t) * np.abs(want) + (2.0 ** -25 if dtype == "f16" else 0.0)).all()
    # in norm such sums are off by 2^-17 of the results at most, 2^-6 of fp16's smallest step of 2^-11: nearly every result is
    # the nearest number of its type (twice 2^-6 for results that are smaller than most)
    nearest = torch.from_numpy(want).to(t)
    assert float((out.cpu() == nearest).double().mean()) > 1 - 2 * 2.0 ** -6
