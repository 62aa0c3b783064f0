"""The layer calls (packed activations, scaled products, weight gradients) against their definitions in 64 bits.

Tolerances.  Packing is exact but for the code's own rounding, which the reference does as well: bits are compared.
Sums of products: inputs that are small integers times powers of two have exact sums in fp32 in every order, and
results are compared to the bit (to the one rounding of the output type); for other inputs a sum of n terms in fp32
is off by at most (n + 4) * 2^-23 times the sum of magnitudes, truncating additions allowed for.  An output
type's rounding is half a step, finfo.eps / 2 of the value.  Activation functions: the functions of the fp32
library are within 16 steps of 2^-23 of their result, and so is each factor: 64 * 2^-24 of max(1, |x|)."""
import math

import numpy as np
import pytest

from tests import layer_reference as ref
from tests.gpu_harness import say

pytestmark = pytest.mark.gpu

TYPES = ["f32", "bf16", "f16"]


def torch_type(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def half_step(t):
    import torch
    return torch.finfo(t).eps / 2


def on_gpu(a, dtype=None, pad_rows=0, front=0, row_gap=0):
    """A dense GPU matrix with the values of `a`: it starts `front` values behind an aligned address and its rows lie
    row_gap values apart; NaN in between, which nothing may read into a result."""
    import torch
    a = np.asarray(a)
    dtype = dtype or torch.float32
    rows, cols = a.shape
    flat = torch.full((front + rows * (cols + row_gap) + 8,), math.nan, dtype=dtype, device="cuda")
    m = flat[front:front + rows * (cols + row_gap)].view(rows, cols + row_gap)[:, :cols]
    m.copy_(torch.from_numpy(np.ascontiguousarray(a)))
    return m


def packed_on_gpu(codes, scales, extra_blocks=0):
    """codes and scales as a packed matrix with garbage where nothing may be read into a result."""
    import torch
    rows, width = codes.shape
    c = torch.full((rows, width + 128 * extra_blocks), 0x7F, dtype=torch.uint8, device="cuda")
    c[:, :width] = torch.from_numpy(codes)
    s = torch.full((rows, -(-scales.shape[1] // 4) * 4 + 4 * extra_blocks), 255, dtype=torch.uint8, device="cuda")
    s[:, :scales.shape[1]] = torch.from_numpy(scales)
    return c, s


def values_in(rows, cols, seed, kind="normal"):
    r = np.random.default_rng([rows, cols, seed])
    if kind == "int":                       # small integers: e4m3 holds them, sums of products are exact
        return r.integers(-4, 5, (rows, cols)).astype(np.float64)
    x = r.standard_normal((rows, cols)) * np.exp(r.standard_normal((1, cols)))
    return x


def special(rows, cols, seed):
    """Blocks of zeros, subnormals, huge and tiny values, infinities, NaN, and maxima at the border 448 * 2^e."""
    r = np.random.default_rng([rows, cols, seed, 9])
    x = (r.standard_normal((rows, cols)) * np.exp2(r.integers(-20, 20, (rows, 1)))).astype(np.float32)
    for b in range(0, cols, 128):
        for row in range(rows):
            k = (row + b // 128) % 9
            v = x[row, b:b + 128]
            if k == 0: v[:] = 0
            elif k == 1: v[:] *= np.float32(1e-43) / max(np.float32(1e-30), np.abs(v).max())
            elif k == 2: v[r.integers(0, len(v))] = np.inf
            elif k == 3: v[r.integers(0, len(v))] = np.nan
            elif k == 4: v[:] = np.clip(v, -400, 400); v[r.integers(0, len(v))] = -448.0
            elif k == 5: v[:] = np.clip(v, -400, 400); v[r.integers(0, len(v))] = np.float32(448.0) * (1 + np.float32(2.0 ** -7))
            elif k == 6: v[r.integers(0, len(v))] = np.finfo(np.float32).max
            elif k == 7: v[:] = -np.inf
    return x


# ---- pack ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_every_16_bit_value_packs_as_defined(dtype):
    """All 65536 bit patterns, each beside one that sets the block's scale."""
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    say(f"layer: pack all values of {dtype}")
    for shift in (0, 3):
        bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(t)
        x = bits.view(512, 128).clone()
        if shift:                            # magnitudes in ascending order would leave small codes untested: mix them
            x = bits[torch.from_numpy(np.random.default_rng(shift).permutation(65536))].view(512, 128).clone()
            x[:, 0] = 2.0 ** shift
        codes, scales = B.alloc_packed(512, 128)
        B.gtopk_pack_rows(x.cuda(), codes, scales)
        want_c, want_s = ref.pack(x.double().numpy())
        assert np.array_equal(scales[:, :1].cpu().numpy(), want_s)
        assert np.array_equal(codes.cpu().numpy(), want_c)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,front,gap", [(1, 1, 0, 0), (1, 128, 0, 0), (3, 127, 1, 0), (5, 129, 3, 2), (2, 1000, 0, 1),
                                                 (17, 300, 7, 5), (33, 2049, 1, 3), (300, 9, 0, 0), (9, 5000, 5, 8)])
def test_pack_rows(dtype, rows, cols, front, gap):
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    for x in (values_in(rows, cols, 1), special(rows, cols, 2)):
        m = on_gpu(x, t, front=front, row_gap=gap)
        nb = -(-cols // 128)
        codes = torch.full((rows, nb * 128 + 128), 0xA5, dtype=torch.uint8, device="cuda")
        scales = torch.full((rows, -(-nb // 4) * 4 + 4), 0xA5, dtype=torch.uint8, device="cuda")
        say(f"layer: pack_rows {dtype} {rows}x{cols} front {front} gap {gap}")
        B.gtopk_pack_rows(m, codes, scales)
        want_c, want_s = ref.pack(m.double().cpu().numpy())
        c, s = codes.cpu().numpy(), scales.cpu().numpy()
        assert np.array_equal(s[:, :nb], want_s)
        assert np.array_equal(c[:, :nb * 128], want_c)
        assert (c[:, nb * 128:] == 0xA5).all() and (s[:, nb:] == 0xA5).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,front,gap", [(1, 1, 0, 0), (128, 128, 0, 0), (1, 300, 1, 0), (300, 1, 0, 0), (129, 127, 3, 1),
                                                 (257, 401, 5, 7), (64, 1024, 0, 0)])
def test_pack_tiles(dtype, rows, cols, front, gap):
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    for x in (values_in(rows, cols, 3), special(rows, cols, 4)):
        m = on_gpu(x, t, front=front, row_gap=gap)
        exact = m.double().cpu().numpy()
        want = [*ref.pack(exact, tiles=True), *ref.pack(exact.T, tiles=True)]
        say(f"layer: pack_tiles {dtype} {rows}x{cols}")
        for both in (True, False):
            out = [*B.alloc_packed(rows, cols), *B.alloc_packed(cols, rows)]
            if both:
                B.gtopk_pack_tiles(m, *out)
            else:
                B.gtopk_pack_tiles(m, *out[:2])
                B.gtopk_pack_tiles(m, None, None, *out[2:])
            for got, exp in zip(out, want):
                assert np.array_equal(got.cpu().numpy()[:, :exp.shape[1]], exp)


# ---- unpack and the activation's backward ---------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
def test_every_code_at_every_scale_unpacks_exactly(dtype):
    """All 256 codes at all 256 scales: one rounding to the type, infinities and NaN where they belong."""
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 2, axis=1)
    c, s = packed_on_gpu(codes, scales, 1)
    out = torch.empty(256, 256, dtype=t, device="cuda")
    say(f"layer: unpack all codes to {dtype}")
    B.gtopk_unpack(c, s, "none", out)
    exact = torch.from_numpy(ref.values(codes, scales, 256))
    want = exact.float().to(t)               # to fp32 the values are exact (or overflow, as in the type)
    got = out.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got.double(), nan=0.0), torch.nan_to_num(want.double(), nan=0.0))


@pytest.mark.parametrize("act", ["none", "relu", "tanh", "sigmoid", "silu", "gelu"])
@pytest.mark.parametrize("dtype,rows,cols,front,gap", [("f32", 1, 1, 0, 0), ("f32", 37, 1001, 1, 2), ("bf16", 5, 4096, 0, 0),
                                                       ("bf16", 33, 129, 3, 1), ("f16", 7, 263, 1, 0)])
def test_activation_and_its_gradient(act, dtype, rows, cols, front, gap):
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    z = values_in(rows, cols, 5) * 3
    z[0, 0] = 0.0
    codes, scales = ref.pack(z)
    x = ref.values(codes, scales, cols)
    c, s = packed_on_gpu(codes, scales, 1)
    dy = on_gpu(values_in(rows, cols, 6), t, front=front, row_gap=gap)
    d = dy.double().cpu().numpy()
    out = on_gpu(np.zeros((rows, cols)), t, front=front, row_gap=gap)
    say(f"layer: {act} {dtype} {rows}x{cols}")
    B.gtopk_unpack(c, s, act, out)
    near = 64 * 2.0 ** -24 * np.maximum(1.0, np.abs(x))
    want = ref.act(act, x)
    # (fp16: values below its normal range are off by half of its smallest step)
    step = half_step(t) * np.abs(want) + (2.0 ** -25 if dtype == "f16" else 0.0)
    assert (np.abs(out.double().cpu().numpy() - want) <= near * (1 + half_step(t)) + step).all()
    dx = on_gpu(np.zeros((rows, cols)), t, front=front + 1, row_gap=gap + 1)
    B.gtopk_activation_grad(c, s, act, dy, dx)
    want = d * ref.slope(act, x)
    step = half_step(t) * np.abs(want) + (2.0 ** -25 if dtype == "f16" else 0.0)
    assert (np.abs(dx.double().cpu().numpy() - want) <= near * np.abs(d) * (1 + half_step(t)) + step).all()
    # the derivative against differences of the function, in 64 bits (slopes change by at most ~1 per unit: h * 2 off)
    if act != "relu":
        h = 1e-5
        differences = (ref.act(act, x + h) - ref.act(act, x - h)) / (2 * h)
        assert np.allclose(ref.slope(act, x), differences, atol=1e-8 + 1e-10 * np.abs(x).max() / h, rtol=1e-8)
    # in place
    B.gtopk_activation_grad(c, s, act, dy, dy)
    assert torch.equal(dy, dx)


@pytest.mark.parametrize("act", ["none", "relu", "tanh", "sigmoid", "silu", "gelu"])
def test_activation_of_far_and_absent_values(act):
    """Largest magnitudes saturate without NaN; a NaN of the checkpoint reaches the result and its gradient, alone."""
    import torch
    from paper_1901_04359_amd import binding as B
    codes = np.zeros((2, 128), np.uint8)
    codes[0, :4] = [0x7E, 0xFE, 0x7F, 0x38]
    codes[1, :4] = [0x7E, 0xFE, 0x7F, 0x38]
    scales = np.array([[247 - 8], [127]], np.uint8)
    c, s = packed_on_gpu(codes, scales)
    x = ref.values(codes, scales, 128)
    out, dx = torch.zeros(2, 128, device="cuda"), torch.zeros(2, 128, device="cuda")
    say(f"layer: {act} of far values")
    B.gtopk_unpack(c, s, act, out)
    B.gtopk_activation_grad(c, s, act, torch.ones(2, 128, device="cuda"), dx)
    for got, want in ((out, ref.act(act, x)), (dx, ref.slope(act, x))):
        g = got.double().cpu().numpy()
        assert np.array_equal(np.isnan(g), np.isnan(want)), act
        fine = ~np.isnan(want)
        assert (np.abs(g - want)[fine] <= 64 * 2.0 ** -24 * np.maximum(1.0, np.abs(want[fine]))).all()


# ---- product ------------------------------------------------------------------------

def int_packed(rows, cols, seed, spread=2):
    """Codes of small integers, with scales that differ by powers of two from block to block: exact sums in fp32."""
    r = np.random.default_rng([rows, cols, seed, 4])
    v = r.integers(-2, 3, (rows, cols)).astype(np.float64)
    nb = -(-cols // 128)
    codes = np.zeros((rows, nb * 128), np.uint8)
    codes[:, :cols] = ref.encode(v)
    scales = r.integers(127 - spread, 127 + spread + 1, (rows, nb)).astype(np.uint8)
    return codes, scales


PRODUCTS = [(1, 1, 1), (1, 4096, 128), (1, 1000, 9216), (2, 17, 129), (3, 64, 127), (16, 16, 128), (17, 33, 260), (5, 2050, 384),
            (64, 64, 1), (63, 130, 640), (128, 128, 256), (129, 257, 1111), (100, 1000, 1025), (256, 256, 512), (255, 513, 2048),
            (300, 520, 130), (520, 1000, 777), (1024, 1025, 136), (33, 31, 20000), (640, 700, 1300)]


@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product_of_integers_is_exact(M, N, K):
    import torch
    from paper_1901_04359_amd import binding as B
    a, b = int_packed(M, K, 1), int_packed(N, K, 2)
    want = ref.values(*a, K) @ ref.values(*b, K).T          # |sum| < 2^24 units of 2^-4
    ga, gb = packed_on_gpu(*a, 1), packed_on_gpu(*b, 2)
    ws = B.alloc_product_workspace(M, N, K)
    ws.fill_(0xA5)
    for dtype in TYPES:
        t = torch_type(dtype)
        for gap in (0, 3):
            out = on_gpu(np.zeros((M, N)), t, front=gap, row_gap=gap)
            flat = out.as_strided((M, N + gap), (N + gap, 1))
            say(f"layer: product {M}x{N}x{K} {dtype} gap {gap}")
            B.gtopk_scaled_product(*ga, *gb, K, out, ws)
            assert torch.equal(out.cpu(), torch.from_numpy(want).float().to(t))
            if gap:
                assert bool(torch.isnan(flat[:, N:]).all())     # what lies between the rows is left alone


@pytest.mark.parametrize("M,N,K", [(1, 300, 5000), (70, 90, 1000), (257, 300, 4096), (513, 770, 2000)])
def test_product_of_activations_and_weights(M, N, K):
    import torch
    from paper_1901_04359_amd import binding as B
    a, b = ref.pack(values_in(M, K, 7)), ref.pack(values_in(N, K, 8) / math.sqrt(K), tiles=True)
    va, vb = ref.values(*a, K), ref.values(*b, K)
    out = torch.zeros(M, N, device="cuda")
    say(f"layer: product {M}x{N}x{K} of real values")
    B.gtopk_scaled_product(*packed_on_gpu(*a), *packed_on_gpu(*b), K, out, B.alloc_product_workspace(M, N, K))
    err = np.abs(out.double().cpu().numpy() - va @ vb.T)
    assert (err <= (K + 4) * 2.0 ** -23 * (np.abs(va) @ np.abs(vb).T)).all()
    # the errors of many sums do not all point the same way: their norm is far below the worst case
    assert np.linalg.norm(err) <= 2.0 ** -17 * np.linalg.norm(va @ vb.T)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K", [(1, 300, 5000), (20, 90, 1000), (70, 90, 1000), (257, 300, 1040), (300, 280, 2000)])
def test_product_rounded_to_16_bits(M, N, K, dtype):
    """Each of eight products of consecutive k loses less than 2^-13 of the largest one's leading bit, the sums of eight add
    up in fp32, and the result is rounded once: 8 * 2^-13 of the largest of every eight, the fp32 sums' bound, half a step."""
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    a, b = ref.pack(values_in(M, K, 7)), ref.pack(values_in(N, K, 8) / math.sqrt(K), tiles=True)
    va, vb = ref.values(*a, K), ref.values(*b, K)
    out = torch.zeros(M, N, dtype=t, device="cuda")
    say(f"layer: product {M}x{N}x{K} to {dtype}")
    B.gtopk_scaled_product(*packed_on_gpu(*a), *packed_on_gpu(*b), K, out, B.alloc_product_workspace(M, N, K))
    want = va @ vb.T
    cut = np.zeros((M, N))
    for k in range(0, K, 8):
        cut += np.abs(va[:, None, k:k + 8] * vb[None, :, k:k + 8]).max(axis=2)
    bound = 8 * 2.0 ** -13 * cut + (K + 4) * 2.0 ** -23 * (np.abs(va) @ np.abs(vb).T)
    err = np.abs(out.double().cpu().numpy() - want)
    assert (err <= bound * (1 + half_step(t)) + half_step(t) * np.abs(want) + (2.0 ** -25 if dtype == "f16" else 0.0)).all()
    # the cut parts have both signs: in norm they stay below the rounding of either type
    assert np.linalg.norm(err) <= 1.1 * half_step(t) * np.linalg.norm(want)


@pytest.mark.parametrize("M,N,K", [(3, 40, 500), (130, 140, 300)])
def test_product_with_nan_and_extreme_scales(M, N, K):
    """A NaN reaches its row or column and nothing else; scales at the ends of their range."""
    import torch
    from paper_1901_04359_amd import binding as B
    a, b = int_packed(M, K, 3), int_packed(N, K, 4)
    a[0][1, 7] = 0x7F                        # a NaN code in row 1 of A, one in column N-1's row of B
    b[0][N - 1, K - 1] = 0xFF
    b[1][N - 2, 0] = 255                     # a NaN scale
    va, vb = ref.values(*a, K), ref.values(*b, K)
    out = torch.zeros(M, N, device="cuda")
    ws = B.alloc_product_workspace(M, N, K)
    say(f"layer: product {M}x{N}x{K} with NaN")
    B.gtopk_scaled_product(*packed_on_gpu(*a), *packed_on_gpu(*b), K, out, ws)
    want = torch.from_numpy(va @ vb.T).float()
    got = out.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    a, b = int_packed(M, K, 3), int_packed(N, K, 4)
    a[1][:], b[1][:] = 1, 247                # 2^-126 * 2^120
    say("layer: product with extreme scales")
    B.gtopk_scaled_product(*packed_on_gpu(*a), *packed_on_gpu(*b), K, out, ws)
    assert torch.equal(out.cpu(), torch.from_numpy(ref.values(*a, K) @ ref.values(*b, K).T).float())


@pytest.mark.parametrize("M,N,K", [(3, 40, 500), (40, 30, 1100), (130, 140, 300)])
@pytest.mark.parametrize("dtype", TYPES)
def test_product_of_scales_over_their_whole_range(M, N, K, dtype):
    """Blocks of every scale that pack makes, in pairs whose product is near 1: sums are exact in every type's path."""
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    a, b = int_packed(M, K, 13), int_packed(N, K, 14)
    r = np.random.default_rng([M, N, K])
    nb = -(-K // 128)
    each = r.integers(7, 248, nb)                             # A's, per block; B's make up for it: 7 .. 247 as well
    a[1][:] = each[None, :]
    b[1][:] = np.clip(254 - each, 7, 247)[None, :]
    want = torch.from_numpy(ref.values(*a, K) @ ref.values(*b, K).T)
    out = torch.zeros(M, N, dtype=t, device="cuda")
    say(f"layer: product {M}x{N}x{K} {dtype}, all scales")
    B.gtopk_scaled_product(*packed_on_gpu(*a), *packed_on_gpu(*b), K, out, B.alloc_product_workspace(M, N, K))
    assert torch.equal(out.cpu(), want.float().to(t))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_product_with_nan_in_16_bits(dtype):
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    for M, N, K in ((3, 40, 500), (130, 140, 300)):
        a, b = int_packed(M, K, 3), int_packed(N, K, 4)
        a[0][1, 7], b[0][N - 1, K - 1], b[1][N - 2, 0] = 0x7F, 0xFF, 255
        out = torch.zeros(M, N, dtype=t, device="cuda")
        say(f"layer: product {M}x{N}x{K} {dtype} with NaN")
        B.gtopk_scaled_product(*packed_on_gpu(*a), *packed_on_gpu(*b), K, out, B.alloc_product_workspace(M, N, K))
        want = torch.from_numpy(ref.values(*a, K) @ ref.values(*b, K).T).float().to(t)
        assert torch.equal(torch.isnan(out.cpu()), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(out.cpu()), torch.nan_to_num(want))


# More than 512 tiles of 128 x 128 but at most 256 of 256 x 256: the product takes the large ones.  One block of 128 to ten, odd
# numbers of them, a tile with a single row, and a single column.
LARGE_PRODUCTS = [(2820, 2851, 1), (2830, 2817, 130), (257, 21890, 300), (2820, 2851, 385), (2945, 2690, 640), (21889, 257, 777), (2817, 2850, 1157)]


def takes_large_tiles(M, N):
    def tiles(side):
        return -(-M // side) * -(-N // side)
    return tiles(128) > 512 and tiles(256) <= 256


@pytest.mark.parametrize("M,N,K", LARGE_PRODUCTS)
def test_large_product_of_integers_is_exact(M, N, K):
    import torch
    from paper_1901_04359_amd import binding as B
    assert takes_large_tiles(M, N)
    a, b = int_packed(M, K, 1), int_packed(N, K, 2)
    want = torch.from_numpy(ref.values(*a, K) @ ref.values(*b, K).T)
    ga, gb = packed_on_gpu(*a, 1), packed_on_gpu(*b, 2)
    ws = B.alloc_product_workspace(M, N, K)
    for dtype in TYPES:
        t = torch_type(dtype)
        flat = torch.full((M * (N + 3) + 8,), math.nan, dtype=t, device="cuda")
        out = flat[3:3 + M * (N + 3)].view(M, N + 3)[:, :N]
        say(f"layer: large product {M}x{N}x{K} {dtype}")
        B.gtopk_scaled_product(*ga, *gb, K, out, ws)
        assert torch.equal(out.cpu(), want.float().to(t))
        assert int(torch.isnan(flat).sum()) == 3 * M + 8            # what lies outside the rows is left alone


def test_large_product_of_real_values():
    """The bounds of the products above, for every 29th row (the bound of what eight products lose takes M N K values)."""
    import torch
    from paper_1901_04359_amd import binding as B
    M, N, K = 2820, 2851, 1100
    a, b = ref.pack(values_in(M, K, 7)), ref.pack(values_in(N, K, 8) / math.sqrt(K), tiles=True)
    va, vb = ref.values(*a, K)[::29], ref.values(*b, K)
    want, size = va @ vb.T, np.abs(va) @ np.abs(vb).T
    cut = np.zeros(want.shape)
    for k in range(0, K, 8):
        cut += np.abs(va[:, None, k:k + 8] * vb[None, :, k:k + 8]).max(axis=2)
    ga, gb = packed_on_gpu(*a), packed_on_gpu(*b)
    for dtype in TYPES:
        t = torch_type(dtype)
        out = torch.zeros(M, N, dtype=t, device="cuda")
        say(f"layer: large product of real values to {dtype}")
        B.gtopk_scaled_product(*ga, *gb, K, out, B.alloc_product_workspace(M, N, K))
        err = np.abs(out[::29].double().cpu().numpy() - want)
        bound = (K + 4) * 2.0 ** -23 * size
        if dtype == "f32":
            assert (err <= bound).all()
            assert np.linalg.norm(err) <= 2.0 ** -17 * np.linalg.norm(want)
        else:
            bound = (8 * 2.0 ** -13 * cut + bound) * (1 + half_step(t)) + half_step(t) * np.abs(want)
            assert (err <= bound + (2.0 ** -25 if dtype == "f16" else 0.0)).all()
            assert np.linalg.norm(err) <= 1.1 * half_step(t) * np.linalg.norm(want)


@pytest.mark.parametrize("dtype", TYPES)
def test_large_product_with_nan_and_every_scale(dtype):
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    M, N, K = 2817, 2850, 640
    a, b = int_packed(M, K, 3), int_packed(N, K, 4)
    each = np.random.default_rng([M, N, K]).integers(7, 248, 5)
    a[1][:] = each[None, :]
    b[1][:] = np.clip(254 - each, 7, 247)[None, :]
    a[0][M - 1, 7], b[0][N - 1, K - 1], b[1][N - 2, 2] = 0x7F, 0xFF, 255
    want = torch.from_numpy(ref.values(*a, K) @ ref.values(*b, K).T).float().to(t)
    out = torch.zeros(M, N, dtype=t, device="cuda")
    say(f"layer: large product {dtype} with NaN and every scale")
    B.gtopk_scaled_product(*packed_on_gpu(*a), *packed_on_gpu(*b), K, out, B.alloc_product_workspace(M, N, K))
    got = out.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


@pytest.mark.parametrize("M,N,far", [(257, 21890, "a"), (21890, 257, "b"), (300, 520, "a")])
def test_product_of_rows_at_the_largest_stride(M, N, far):
    """A tile's last row begins 255 * 2^23 bytes behind its first one, of large tiles and of small ones."""
    import torch
    from paper_1901_04359_amd import binding as B
    K = 300
    a, b = int_packed(M, K, 5), int_packed(N, K, 6)
    want = torch.from_numpy(ref.values(*a, K) @ ref.values(*b, K).T).float()
    ga, gb = packed_on_gpu(*a), packed_on_gpu(*b)
    near = ga if far == "a" else gb
    wide = []
    for t in near:
        w = torch.empty(t.shape[0] * 2 ** 23, dtype=torch.uint8, device="cuda").view(t.shape[0], 2 ** 23)[:, :t.shape[1]]
        w.copy_(t)
        wide.append(w)
    ga, gb = (wide, gb) if far == "a" else (ga, wide)
    ws = B.alloc_product_workspace(M, N, K)
    for dtype in TYPES:
        out = torch.zeros(M, N, dtype=torch_type(dtype), device="cuda")
        say(f"layer: product {M}x{N}x{K} {dtype}, rows 2^23 bytes apart")
        B.gtopk_scaled_product(*ga, *gb, K, out, ws)
        assert torch.equal(out.cpu(), want.to(torch_type(dtype)))


# ---- weight gradient ------------------------------------------------------------------

def begins(P, rows, kind, seed=0):
    if kind == "even":
        return [rows // P * w for w in range(P + 1)]
    r = np.random.default_rng([P, rows, seed])
    cuts = np.sort(r.integers(0, rows + 1, P + 1))           # rows before the first and behind the last belong to nobody
    if kind == "ragged":
        cuts[0], cuts[-1] = 0, rows
    return [int(c) for c in cuts]


GRADS = [(1, 1, 1, 1, "even"), (1, 1, 5, 300, "even"), (4, 4, 3, 2, "even"), (2, 64, 16, 16, "even"), (8, 8, 130, 129, "even"),
         (3, 33, 17, 40, "ragged"), (4, 100, 64, 128, "loose"), (2, 500, 128, 128, "even"), (1, 2000, 100, 260, "even"),
         (5, 77, 257, 385, "ragged"), (1, 9000, 33, 65, "even"), (8, 1501, 100, 131, "ragged"), (16, 1024, 256, 130, "even"),
         (1, 0, 20, 30, "even"), (6, 3, 9, 140, "loose"), (32, 32 * 40, 40, 200, "even"),
         (3, 70, 40, 512, "ragged"), (2, 300, 130, 1024, "even"), (4, 64, 33, 544, "even"), (1, 33, 20, 640, "even"),
         (2, 6000, 1000, 1100, "ragged"), (3, 4700, 1025, 770, "loose"), (1, 9001, 1030, 900, "even")]


@pytest.mark.parametrize("P,rows,N,K,kind", GRADS)
@pytest.mark.parametrize("dtype", TYPES)
def test_weight_grad_of_integers_is_exact(P, rows, N, K, kind, dtype):
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    codes, scales = int_packed(rows, K, 5)
    r = np.random.default_rng([P, rows, N, K])
    # values with as many significant bits as the sums leave room for (fp32: 2^10 * 2^4 * 2^... < 2^24 of the smallest unit)
    top = {"f32": 2 ** 6 if rows > 512 else 2 ** 9, "bf16": 16, "f16": 64}[dtype]
    dy = r.integers(-top, top + 1, (rows, N)).astype(np.float64)
    begin = begins(P, rows, kind)
    want = ref.weight_grad(dy, ref.values(codes, scales, K), begin)
    assert np.abs(want).max(initial=0) < 2 ** 22             # units of 2^-2: below 2^24
    behind = 5
    grads = torch.full((P, behind + N * K + 3), 7.0, device="cuda")
    grad = grads[:, behind:behind + N * K].unflatten(1, (N, K))
    d = on_gpu(dy, t, front=1, row_gap=3) if rows else torch.zeros(0, N, dtype=t, device="cuda")
    c, s = packed_on_gpu(codes, scales, 1)
    plan = None if kind == "even" else torch.tensor(begin, dtype=torch.int32, device="cuda")
    ws = B.alloc_weight_grad_workspace(rows, P, N, K)
    ws.fill_(0xFF)
    say(f"layer: weight_grad {dtype} P {P} rows {rows} {N}x{K} {kind}")
    B.gtopk_weight_grad(d, c, s, plan, grad, False, ws)
    w32 = torch.from_numpy(want).float()
    assert torch.equal(grad.cpu(), w32)
    B.gtopk_weight_grad(d, c, s, plan, grad, True, ws)
    assert torch.equal(grad.cpu(), 2 * w32)
    assert bool((grads[:, :behind] == 7.0).all()) and bool((grads[:, behind + N * K:] == 7.0).all())


@pytest.mark.parametrize("behind,gap", [(0, 0), (32, 32), (1, 0), (31, 1), (7, 25), (16, 8), (30, 3), (100, 28)])
@pytest.mark.parametrize("K", [512, 608, 1152, 96])
def test_weight_grad_wherever_rows_begin(behind, gap, K):
    """dW anywhere in the workers' rows, in front of and behind other layers: tiles follow memory lines, sums do not."""
    import torch
    from paper_1901_04359_amd import binding as B
    P, T, N = 3, 45, 37
    codes, scales = int_packed(P * T, K, 31)
    dy = np.random.default_rng([behind, K]).integers(-8, 9, (P * T, N)).astype(np.float64)
    want = torch.from_numpy(ref.weight_grad(dy, ref.values(codes, scales, K), [0, T, 2 * T, 3 * T])).float()
    base = torch.full((64 + P * (behind + N * K + gap) + 64,), 7.0, device="cuda")
    assert base.data_ptr() % 128 == 0
    grads = base[64:-64].view(P, behind + N * K + gap)
    grad = grads[:, behind:behind + N * K].unflatten(1, (N, K))
    ws = B.alloc_weight_grad_workspace(P * T, P, N, K)
    c, s = packed_on_gpu(codes, scales)
    say(f"layer: weight_grad behind {behind} gap {gap} K {K}")
    for dtype in TYPES:
        d = on_gpu(dy, torch_type(dtype))
        B.gtopk_weight_grad(d, c, s, None, grad, False, ws)
        assert torch.equal(grad.cpu(), want)
        B.gtopk_weight_grad(d, c, s, None, grad, True, ws)
        assert torch.equal(grad.cpu(), 2 * want)
        rest = base.clone()
        rest[64:-64].view(P, -1)[:, behind:behind + N * K] = 7.0
        assert bool((rest == 7.0).all())


@pytest.mark.parametrize("P,rows,N,K,kind", [(4, 300, 70, 200, "ragged"), (1, 5000, 130, 140, "even"), (16, 16, 64, 300, "even")])
@pytest.mark.parametrize("dtype", TYPES)
def test_weight_grad_of_activations(P, rows, N, K, kind, dtype):
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    codes, scales = ref.pack(np.maximum(values_in(rows, K, 11), 0))
    x = ref.values(codes, scales, K)
    d = on_gpu(values_in(rows, N, 12) * 1e-3, t)
    dy = d.double().cpu().numpy()
    begin = begins(P, rows, kind)
    grad = torch.empty(P, N, K, device="cuda")
    plan = torch.tensor(begin, dtype=torch.int32, device="cuda")
    say(f"layer: weight_grad {dtype} P {P} rows {rows} {N}x{K} of real values")
    B.gtopk_weight_grad(d, *packed_on_gpu(codes, scales), plan, grad, False, B.alloc_weight_grad_workspace(rows, P, N, K))
    got, want = grad.double().cpu().numpy(), ref.weight_grad(dy, x, begin)
    size = ref.weight_grad(np.abs(dy), np.abs(x), begin)
    n = np.diff(begin)[:, None, None]
    parts = {"bf16": 1, "f16": 2, "f32": 3}[dtype]           # terms per product
    # (2^-126: the parts of a value that may be taken as 0, times the largest x)
    assert (np.abs(got - want) <= (parts * n + 4) * 2.0 ** -23 * size + n * 2.0 ** -126 * np.abs(x).max(initial=0)).all()
    assert np.linalg.norm(got - want) <= 2.0 ** -18 * np.linalg.norm(want)
    again = torch.empty_like(grad)
    B.gtopk_weight_grad(d, *packed_on_gpu(codes, scales), plan, again, False, B.alloc_weight_grad_workspace(rows, P, N, K))
    assert torch.equal(grad, again)                          # the same sums in the same order


@pytest.mark.parametrize("dtype", TYPES)
def test_weight_grad_of_values_that_are_not_finite(dtype):
    """inf and NaN of dY reach their row of the worker's gradient; the checkpoint's NaN its column; workers stay apart."""
    import torch
    from paper_1901_04359_amd import binding as B
    t = torch_type(dtype)
    P, T, N, K = 3, 40, 20, 150
    codes, scales = int_packed(P * T, K, 6, spread=0)
    codes[codes == 0] = 0x38                                  # no zeros: inf * 0 would be NaN
    codes[codes == 0x80] = 0x38
    codes[:, K:] = 0
    codes[T + 3, 140] = 0x7F
    dy = np.ones((P * T, N))
    dy[5, 4], dy[2 * T + 1, 0], dy[2 * T + 2, 1] = np.inf, np.nan, -np.inf
    grad = torch.empty(P, N, K, device="cuda")
    say(f"layer: weight_grad {dtype} not finite")
    B.gtopk_weight_grad(on_gpu(dy, t), *packed_on_gpu(codes, scales), None, grad, False, B.alloc_weight_grad_workspace(P * T, P, N, K))
    want = torch.from_numpy(ref.weight_grad(dy, ref.values(codes, scales, K), [0, T, 2 * T, 3 * T])).float()
    got = grad.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


def test_weight_grad_keeps_every_bit_of_fp32():
    """Values with all 24 bits set, tiny and huge ones: dY enters exactly."""
    import torch
    from paper_1901_04359_amd import binding as B
    codes, scales = np.zeros((1, 128), np.uint8), np.full((1, 1), 127, np.uint8)
    codes[0, :3] = ref.encode(np.array([1.0, 2.0, 0.5]))
    bits = np.random.default_rng(5).integers(0x10800000, 0x7E000000, 500, dtype=np.int64).astype(np.uint32)
    dy = bits.view(np.float32).astype(np.float64)[None, :]
    grad = torch.empty(1, 500, 3, device="cuda")
    say("layer: weight_grad keeps fp32")
    B.gtopk_weight_grad(on_gpu(dy), *packed_on_gpu(codes, scales), None, grad, False, B.alloc_weight_grad_workspace(1, 1, 500, 3))
    assert torch.equal(grad[0].cpu(), torch.from_numpy(dy.T * np.array([1.0, 2.0, 0.5])).float())


def test_row_begin_out_of_range_stays_inside():
    """Entries that are no row numbers are clamped: no read outside the matrices, no write outside the gradients."""
    import torch
    from paper_1901_04359_amd import binding as B
    rows, N, K = 30, 20, 140
    codes, scales = int_packed(rows, K, 8)
    dy = np.random.default_rng(8).integers(-4, 5, (rows, N)).astype(np.float64)
    plan = torch.tensor([-5, 10, 7, 2**31 - 1, -2**31], dtype=torch.int32, device="cuda")
    grad = torch.full((4, N, K), 7.0, device="cuda")
    say("layer: weight_grad, row_begin out of range")
    B.gtopk_weight_grad(on_gpu(dy), *packed_on_gpu(codes, scales), plan, grad, False, B.alloc_weight_grad_workspace(rows, 4, N, K))
    x = ref.values(codes, scales, K)
    want = np.stack([dy[a:b].T @ x[a:b] for a, b in ((0, 10), (10, 10), (7, 30), (30, 30))])
    assert torch.equal(grad.cpu(), torch.from_numpy(want).float())


def test_offsets_past_32_bits():
    """Matrices of more than 2^32 bytes, gradient rows more than 2^32 bytes apart: the far ends against the near ones."""
    import torch
    from paper_1901_04359_amd import binding as B
    rows, cols, tail = 560_000, 8192, 130
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    codes, scales = B.alloc_packed(rows, cols)
    assert codes.numel() > 2**32
    say("layer: pack past 2^32")
    B.gtopk_pack_rows(x, codes, scales)
    want_c, want_s = ref.pack(x[-tail:].double().cpu().numpy())
    assert np.array_equal(codes[-tail:].cpu().numpy(), want_c) and np.array_equal(scales[-tail:].cpu().numpy(), want_s)
    far, near = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda"), torch.empty(tail, cols, dtype=torch.bfloat16, device="cuda")
    c, s = codes[-tail:].clone(), scales[-tail:].clone()
    say("layer: unpack and gradient past 2^32")
    B.gtopk_unpack(codes, scales, "silu", far)
    B.gtopk_unpack(c, s, "silu", near)
    assert torch.equal(far[-tail:], near)
    B.gtopk_activation_grad(codes, scales, "silu", x, x)
    dy = torch.empty(tail, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    far[-tail:] = dy
    B.gtopk_activation_grad(c, s, "silu", dy, near)
    B.gtopk_activation_grad(codes, scales, "silu", far, far)
    assert torch.equal(far[-tail:], near)
    del far, near, x
    b = B.alloc_packed(40, cols)
    B.gtopk_pack_rows(torch.empty(40, cols, device="cuda").normal_(generator=gen), *b)
    say("layer: product past 2^32")
    out, part = torch.empty(rows, 40, device="cuda"), torch.empty(tail, 40, device="cuda")
    B.gtopk_scaled_product(codes, scales, *b, cols, out, B.alloc_product_workspace(rows, 40, cols))
    B.gtopk_scaled_product(c, s, *b, cols, part, B.alloc_product_workspace(tail, 40, cols))
    size = part.abs().max()
    assert bool(((out[-tail:] - part).abs() <= cols * 2.0 ** -22 * size).all())      # the near one is summed in shares of K
    # the last rows as one of three workers, whose gradients lie 6 GB apart
    N = 12
    d = torch.empty(rows, N, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    grads = torch.empty(3, 1_500_000_000, device="cuda")
    grad = grads[:, 7:7 + N * cols].unflatten(1, (N, cols))
    plan = torch.tensor([0, 100, 100, rows], dtype=torch.int32, device="cuda")
    plan[2] = rows - tail
    say("layer: weight_grad past 2^32")
    B.gtopk_weight_grad(d, codes, scales, plan, grad, False, B.alloc_weight_grad_workspace(rows, 3, N, cols))
    one = torch.empty(1, N, cols, device="cuda")
    B.gtopk_weight_grad(d[-tail:], c, s, None, one, False, B.alloc_weight_grad_workspace(tail, 1, N, cols))
    size = one.abs().max()
    assert bool(((grad[2] - one[0]).abs() <= tail * 2.0 ** -22 * size).all())
    want = d[:100].float().t() @ (codes[:100].view(torch.float8_e4m3fn).float() *
                                  torch.exp2(scales[:100, :cols // 128].float() - 127).repeat_interleave(128, dim=1))
    assert bool(((grad[0] - want).abs() <= 200 * 2.0 ** -22 * want.abs().max()).all())


def test_more_rows_and_jobs_than_blocks_in_a_launch():
    """Grids are capped: blocks walk the rows, and the workers' tiles, that are left."""
    import torch
    from paper_1901_04359_amd import binding as B
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    rows, cols = 2_200_000, 9                                # 65535 blocks of 16 or 32 rows, and 100,000 rows more
    for t in (torch.float32, torch.bfloat16):
        x = torch.empty(rows, cols, device="cuda").normal_(generator=gen).to(t)
        codes, scales = B.alloc_packed(rows, cols)
        out = torch.zeros_like(x)
        say(f"layer: {rows} rows of {cols}")
        B.gtopk_pack_rows(x, codes, scales)
        B.gtopk_unpack(codes, scales, "none", out)
        assert bool(((out - x).float().abs() <= x.float().abs().amax(dim=1, keepdim=True) * 2.0 ** -4).all())
        for at in (0, 1_048_500, 2_097_100, rows - 60):
            want = ref.values(*ref.pack(x[at:at + 60].double().cpu().numpy()), cols)
            assert np.array_equal(out[at:at + 60].double().cpu().numpy(), want)
        B.gtopk_activation_grad(codes, scales, "relu", x, x)
        assert torch.equal(x, torch.where(out > 0, x, torch.zeros_like(x)))
        del x, out, codes, scales
    P, K = 32768, 130 * 128                                  # 4.26 million tiles
    x = torch.randint(-4, 5, (P, K), device="cuda", generator=gen, dtype=torch.int32).to(torch.bfloat16)
    codes, scales = B.alloc_packed(P, K)
    B.gtopk_pack_rows(x, codes, scales)
    dy = torch.randint(-8, 9, (P, 1), device="cuda", generator=gen, dtype=torch.int32).to(torch.bfloat16)
    grad = torch.empty(P, 1, K, device="cuda")
    say("layer: weight_grad of 32768 workers")
    B.gtopk_weight_grad(dy, codes, scales, None, grad, False, B.alloc_weight_grad_workspace(P, P, 1, K))
    assert torch.equal(grad[:, 0], dy.float() * x.float())


# ---- together, on streams, in graphs --------------------------------------------------

class Layers:
    """Two layers of P workers, forward and backward by the calls under test, then the step and the update."""

    def __init__(self, P, T, sizes, k, seed=0):
        import torch
        from paper_1901_04359_amd import binding as B
        self.B, self.P, self.T, self.sizes, self.k = B, P, T, sizes, k
        d0, d1, d2 = sizes
        self.at = [3, 3 + d1 * d0]                            # an odd place of the flat row
        self.m = self.at[1] + d2 * d1 + 2
        r = np.random.default_rng([P, T, *sizes, seed])
        w = r.standard_normal(self.m) * 0.05
        self.weights = torch.from_numpy(w).float().cuda()
        self.x0 = on_gpu(r.standard_normal((P * T, d0)))
        self.target = on_gpu(r.standard_normal((P * T, d2)))
        zeros = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")
        self.grads, self.residual = zeros(P, self.m), zeros(P, self.m)
        R = P * T
        self.cx, self.cz, self.ch, self.cd = (B.alloc_packed(R, n) for n in (d0, d1, d1, d2))
        self.w0, self.w1, self.w1t = B.alloc_packed(d1, d0), B.alloc_packed(d2, d1), B.alloc_packed(d1, d2)
        self.z, self.h, self.dz, self.y, self.dy = zeros(R, d1), zeros(R, d1), zeros(R, d1), zeros(R, d2), zeros(R, d2)
        self.ws = [B.alloc_product_workspace(R, a, b) for a, b in ((d1, d0), (d2, d1), (d1, d2))]
        self.wg = [B.alloc_weight_grad_workspace(R, P, d1, d0), B.alloc_weight_grad_workspace(R, P, d2, d1)]
        self.g_idx, self.g_val = zeros(k, dtype=torch.int32), zeros(k)
        self.step_ws = B.alloc_workspace(self.m, k, P)

    def layer(self, flat, i):
        n, kk = self.sizes[i + 1], self.sizes[i]
        at = self.at[i]
        return flat[..., at:at + n * kk].unflatten(-1, (n, kk))

    def backward(self):
        B, (d0, d1, d2) = self.B, self.sizes
        B.gtopk_pack_tiles(self.layer(self.weights, 0), *self.w0)
        B.gtopk_pack_tiles(self.layer(self.weights, 1), *self.w1, *self.w1t)
        B.gtopk_pack_rows(self.x0, *self.cx)
        B.gtopk_scaled_product(*self.cx, *self.w0, d0, self.z, self.ws[0])
        B.gtopk_pack_rows(self.z, *self.cz)                   # the checkpoint: what goes into the activation
        B.gtopk_unpack(*self.cz, "gelu", self.h)
        B.gtopk_pack_rows(self.h, *self.ch)
        B.gtopk_scaled_product(*self.ch, *self.w1, d1, self.y, self.ws[1])
        self.dy.copy_(self.y).sub_(self.target)               # the gradient of half the squared distance
        B.gtopk_pack_rows(self.dy, *self.cd)
        B.gtopk_weight_grad(self.dy, *self.ch, None, self.layer(self.grads, 1), False, self.wg[1])
        B.gtopk_scaled_product(*self.cd, *self.w1t, d2, self.dz, self.ws[2])
        B.gtopk_activation_grad(*self.cz, "gelu", self.dz, self.dz)
        B.gtopk_weight_grad(self.dz, *self.cx, None, self.layer(self.grads, 0), False, self.wg[0])

    def step(self):
        self.B.gtopk_step(self.grads, self.residual, self.k, self.g_idx, self.g_val, None, None, self.step_ws)
        self.B.gtopk_apply_update(self.weights, self.k, self.g_idx, self.g_val, 0.01)


def test_an_iteration_from_samples_to_updated_weights():
    """Forward, backward, step and update in a row: every stage against 64 bits on what the stage before it left,
    the step against the oracle."""
    import torch
    from oracle import gtopk_oracle as orc
    net = Layers(4, 24, (200, 150, 70), 300)
    d0, d1, d2 = net.sizes
    res = np.zeros((net.P, net.m), np.float32)
    for it in range(2):
        before = net.weights.clone()
        say(f"layer: iteration {it}")
        net.backward()
        net.step()
        torch.cuda.synchronize()
        num = lambda t: t.double().cpu().numpy()
        pk = lambda p: (p[0].cpu().numpy(), p[1].cpu().numpy())
        val = lambda p, cols: ref.values(pk(p)[0], pk(p)[1][:, :-(-cols // 128)], cols)
        w0, w1 = num(net.layer(before, 0)), num(net.layer(before, 1))
        for p, exact, cols, tiles in ((net.w0, w0, d0, True), (net.w1, w1, d1, True), (net.w1t, w1.T, d2, True), (net.cx, num(net.x0), d0, False),
                                      (net.cz, num(net.z), d1, False), (net.ch, num(net.h), d1, False), (net.cd, num(net.dy), d2, False)):
            assert np.array_equal(val(p, cols), ref.values(*ref.pack(exact, tiles), cols))
        def close(got, want, size, n):
            assert (np.abs(num(got) - want) <= (n + 4) * 2.0 ** -23 * size).all()
        close(net.z, val(net.cx, d0) @ val(net.w0, d0).T, np.abs(val(net.cx, d0)) @ np.abs(val(net.w0, d0)).T, d0)
        close(net.y, val(net.ch, d1) @ val(net.w1, d1).T, np.abs(val(net.ch, d1)) @ np.abs(val(net.w1, d1)).T, d1)
        back = val(net.cd, d2) @ val(net.w1t, d2).T
        size = np.abs(val(net.cd, d2)) @ np.abs(val(net.w1t, d2)).T
        z = val(net.cz, d1)
        bound = (d2 + 4) * 2.0 ** -23 * size * 1.2 + 65 * 2.0 ** -24 * np.maximum(1, np.abs(z)) * np.abs(back) * 1.2
        assert (np.abs(num(net.dz) - back * ref.slope("gelu", z)) <= bound).all()
        begin = [net.T * w for w in range(net.P + 1)]
        for i, (d, x) in enumerate(((num(net.dz), val(net.cx, d0)), (num(net.dy), val(net.ch, d1)))):
            close(net.layer(net.grads, i), ref.weight_grad(d, x, begin), ref.weight_grad(np.abs(d), np.abs(x), begin), 3 * net.T)
        g = net.grads.cpu().numpy()
        assert (g[:, :3] == 0).all() and (g[:, -2:] == 0).all()
        exp = orc.step(res, g, net.k)
        res = exp["residual"]
        assert np.array_equal(net.g_idx.cpu().numpy().view(np.uint32), exp["g_idx"])
        assert np.array_equal(net.g_val.cpu().numpy(), exp["g_val"]) and np.array_equal(net.residual.cpu().numpy(), res)
        w = before.cpu().numpy()
        w[exp["g_idx"]] -= np.float32(0.01) * exp["g_val"]
        assert np.array_equal(net.weights.cpu().numpy(), w)


def test_weight_grad_against_differences():
    """sum(dY * (X W^T)) is linear in W: its differences in 64 bits are the gradient."""
    import torch
    from paper_1901_04359_amd import binding as B
    rows, N, K = 50, 6, 40
    codes, scales = ref.pack(values_in(rows, K, 21))
    x, dy = ref.values(codes, scales, K), values_in(rows, N, 22).astype(np.float32).astype(np.float64)
    grad = torch.empty(1, N, K, device="cuda")
    say("layer: weight_grad against differences")
    B.gtopk_weight_grad(on_gpu(dy), *packed_on_gpu(codes, scales), None, grad, False, B.alloc_weight_grad_workspace(rows, 1, N, K))
    w = values_in(N, K, 23)
    loss = lambda w: float((dy * (x @ w.T)).sum())
    for n, k in ((0, 0), (5, 39), (3, 17)):
        e = np.zeros((N, K))
        e[n, k] = 0.5
        size = (np.abs(dy[:, n]) * np.abs(x[:, k])).sum()
        assert abs((loss(w + e) - loss(w - e)) - float(grad[0, n, k])) <= (3 * rows + 4) * 2.0 ** -23 * size + 1e-9


def test_on_another_stream_and_in_a_graph():
    """The calls follow the current stream; captured, they replay with the same results, between eager work on the same
    and on other buffers."""
    import torch
    net = Layers(2, 33, (130, 260, 40), 50, seed=3)
    say("layer: eager")
    net.backward()
    torch.cuda.synchronize()
    want = net.grads.clone()
    side = torch.cuda.Stream()
    net.grads.zero_()
    side.wait_stream(torch.cuda.current_stream())
    say("layer: side stream")
    with torch.cuda.stream(side):
        net.backward()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(net.grads, want)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    say("layer: capture")
    with torch.cuda.graph(graph):
        net.backward()
    other = Layers(2, 33, (130, 260, 40), 50, seed=4)
    for i in range(4):
        net.grads.zero_()
        say(f"layer: replay {i}")
        graph.replay()
        other.backward()
        torch.cuda.synchronize()
        assert torch.equal(net.grads, want)
        if i == 1:                           # new inputs in the captured buffers
            net.x0.mul_(0.5)
            graph.replay()
            torch.cuda.synchronize()
            replayed = net.grads.clone()
            net.backward()
            assert torch.equal(net.grads, replayed) and not torch.equal(replayed, want)
            net.x0.mul_(2.0)


def test_shapes_that_do_not_fit_are_refused():
    import torch
    from paper_1901_04359_amd import binding as B
    x = torch.zeros(4, 130, device="cuda")
    c, s = B.alloc_packed(4, 130)
    c2, s2 = B.alloc_packed(4, 300)
    ws = B.alloc_product_workspace(4, 4, 300)
    out = torch.full((4, 4), 7.0, device="cuda")
    with pytest.raises(ValueError):
        B.gtopk_pack_rows(x[:3], c, s)
    with pytest.raises(ValueError):
        B.gtopk_pack_rows(x.t(), c, s)
    with pytest.raises(ValueError):
        B.gtopk_pack_tiles(x, c, s, c, s)
    with pytest.raises(ValueError):
        B.gtopk_pack_tiles(x, c, None)
    with pytest.raises(ValueError):
        B.gtopk_activation_grad(c, s, "relu", x, x[:, :100])
    with pytest.raises(ValueError):
        B.gtopk_scaled_product(c, s, c2, s2, 300, out, ws)
    with pytest.raises(B.GtopkError) as err:
        B.gtopk_scaled_product(c2, s2, c2, s2, 300, out, ws[:16])
    assert err.value.status == B.GTOPK_EWORKSPACE
    with pytest.raises(ValueError):
        B.gtopk_weight_grad(x, c, s, None, torch.zeros(2, 130, 131, device="cuda")[:, :, :130], False, ws)
    with pytest.raises(ValueError):
        B.gtopk_weight_grad(x, c, s, torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 130, 130, device="cuda"), False, ws)
    with pytest.raises(B.GtopkError):
        B.gtopk_weight_grad(x, c, s, None, torch.zeros(3, 130, 130, device="cuda"), False, B.alloc_weight_grad_workspace(4, 3, 130, 130))
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
