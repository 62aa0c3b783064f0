"""Weight gradients at the sizes that decide which tiles they take: results that are written along memory lines, large tiles without shares
of the rows, bands of tiles, and sums over most of a long batch.  The rules are written out here as well (`plan`), so that a
change to them does not silently leave a kernel without its test.

Inputs are small integers, sums are exact in fp32 in every order, and the results are compared to the bit."""
import numpy as np
import pytest

from tests import layer_reference as ref
from tests.gpu_harness import say
from tests.test_gpu_layer import TYPES, torch_type

pytestmark = pytest.mark.gpu

PARTS = {"bf16": 1, "f16": 2, "f32": 3}


def cdiv(a, b):
    return -(-a // b)


def tiles_of(side, P, rows, N, K):
    """(tiles, shares of the rows) with tiles of this side"""
    tiles = cdiv(N, side) * cdiv(K, side) * P
    shares = max(1, min(rows // P // (1024 if side == 256 else 256), (256 if side == 256 else 512) // tiles))
    return tiles, shares


def plan(dtype, P, rows, N, K, aligned):
    """(kernel, shares of the rows) that a weight gradient takes; aligned: every row of dW begins with a memory line of 128 bytes"""
    each = rows // P
    small, shares = tiles_of(128, P, rows, N, K)
    if dtype == "bf16" and each >= 512:
        large, large_shares = tiles_of(256, P, rows, N, K)
        if large_shares == 1:
            gain = 7 * cdiv(large, 256) <= 2 * cdiv(small * shares, 256)
        else:
            gain = large * large_shares >= 192 and (shares > 1 or each // large_shares >= 2048)
        if gain:
            return "large", large_shares
    if K % 32 == 0 and each * PARTS[dtype] <= 256 and P * N * K >= 2 ** 26:
        if aligned or (each <= 128 and K >= 1024 if dtype == "bf16" else each * PARTS[dtype] <= 64 and K >= 4096):
            return "lines", shares
    return ("small" if dtype == "bf16" else "wide"), shares


def integer_case(P, rows, N, K, dtype, seed=0):
    """dY [rows][N] and X [rows][K] of small integers on the GPU, X also packed"""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000 * P + 10 * rows + seed)
    dy = torch.randint(-3, 4, (rows, N), device="cuda", generator=gen, dtype=torch.int32).to(torch_type(dtype))
    x = torch.randint(-2, 3, (rows, K), device="cuda", generator=gen, dtype=torch.int64)
    nb = cdiv(K, 128)
    codes = torch.zeros(rows, nb * 128, dtype=torch.uint8, device="cuda")
    codes[:, :K] = torch.from_numpy(ref.encode(np.arange(-2.0, 3.0))).cuda()[x + 2]
    scales = torch.randint(126, 129, (rows, cdiv(nb, 4) * 4), device="cuda", generator=gen, dtype=torch.int32).to(torch.uint8)
    f = torch.exp2(scales[:, :nb].double() - 127.0).repeat_interleave(128, dim=1)[:, :K]
    return dy, codes, scales, x.double() * f


def check(P, rows, N, K, dtype, behind, gap, begin=None, again=True):
    """Into rows of 7s, `behind` values behind their start and `gap` before the next; then onto what is there."""
    import torch
    from paper_1901_04359_amd import binding as B
    dy, codes, scales, x = integer_case(P, rows, N, K, dtype)
    at = begin or [rows // P * w for w in range(P + 1)]
    base = torch.full((32 + P * (behind + N * K + gap) + 32,), 7.0, device="cuda")
    assert base.data_ptr() % 128 == 0
    inside = base[32:-32].view(P, behind + N * K + gap)
    grad = inside[:, behind:behind + N * K].unflatten(1, (N, K))
    ws = B.alloc_weight_grad_workspace(rows, P, N, K)
    ws.fill_(0xFF)
    row_begin = None if begin is None else torch.tensor(begin, dtype=torch.int32, device="cuda")
    say(f"layer: weight_grad {dtype} P {P} rows {rows} {N}x{K} behind {behind} gap {gap}")
    for times in (1, 2) if again else (1,):
        B.gtopk_weight_grad(dy, codes, scales, row_begin, grad, times == 2, ws)
        for w in range(P):
            want = (dy[at[w]:at[w + 1]].double().t().contiguous() @ x[at[w]:at[w + 1]]).mul_(times)
            assert float(want.abs().max()) < 2 ** 23
            assert torch.equal(grad[w], want.float()), (w, times)
        assert bool((base[:32] == 7.0).all()) and bool((base[-32:] == 7.0).all())
        assert bool((inside[:, :behind] == 7.0).all()) and bool((inside[:, behind + N * K:] == 7.0).all())


# ---- results written along memory lines -------------------------------------------------

@pytest.mark.parametrize("P,T,N,K,behind,gap", [
    (64, 45, 1021, 1056, 0, 0), (64, 45, 1021, 1056, 1, 0), (64, 30, 1021, 1056, 31, 1), (63, 33, 1021, 1152, 7, 25), (3, 100, 5500, 4128, 16, 8),
    (2, 3, 8200, 4224, 30, 3), (1, 64, 16400, 4096, 100, 28), (1024, 2, 64, 1024, 5, 0), (260, 17, 512, 512, 0, 0), (3000, 1, 700, 32, 32, 64)])
@pytest.mark.parametrize("dtype", TYPES)
def test_large_results_wherever_rows_begin(P, T, N, K, behind, gap, dtype):
    aligned = behind % 32 == 0 and (behind + N * K + gap) % 32 == 0
    few = T * PARTS[dtype] <= 64
    expected = "lines" if T * PARTS[dtype] <= 256 and (aligned or (K >= 1024 if dtype == "bf16" else few and K >= 4096)) else None
    assert (plan(dtype, P, P * T, N, K, aligned)[0] == "lines") == (expected == "lines")
    check(P, P * T, N, K, dtype, behind, gap)


def test_large_result_of_uneven_shares():
    """One worker without rows, one with most of them, some rows that nobody has: along lines from an odd place."""
    P, rows, N, K = 16, 640, 1100, 4096
    begin = [0, 0, 5, 400, 400] + [400 + 17 * i for i in range(1, 13)]
    assert plan("bf16", P, rows, N, K, False)[0] == "lines"
    check(P, rows, N, K, "bf16", 9, 3, begin)


# ---- large tiles without shares of the rows -----------------------------------------------

@pytest.mark.parametrize("P,rows,N,K,behind,gap", [(1, 513, 4096, 4096, 0, 0), (1, 600, 4090, 3850, 5, 3), (1, 512, 3585, 3841, 32, 0), (2, 2500, 2816, 2816, 0, 64),
                                                   (4, 2049 * 4, 1800, 2040, 7, 0), (8, 8 * 545, 2000, 2048, 31, 1)])
def test_large_tiles_without_shares(P, rows, N, K, behind, gap):
    assert plan("bf16", P, rows, N, K, behind == 0) == ("large", 1)
    check(P, rows, N, K, "bf16", behind, gap)


def test_large_tiles_of_uneven_shares():
    P, rows, N, K = 4, 2400, 1900, 2048
    assert plan("bf16", P, rows, N, K, False) == ("large", 1)
    check(P, rows, N, K, "bf16", 11, 2, [3, 3, 40, 2040, 2399])


@pytest.mark.parametrize("P,rows,N,K,shares", [(1, 16384, 1000, 1024, 16), (2, 10000, 1024, 1800, 4), (1, 5000, 2048, 4000, 2)])
def test_large_tiles_in_shares(P, rows, N, K, shares):
    assert plan("bf16", P, rows, N, K, False) == ("large", shares)
    check(P, rows, N, K, "bf16", 3, 1)


# ---- scales from the smallest on, and NaN, in the kernels that only large sizes take --------

@pytest.mark.parametrize("kernel,P,rows,N,K,behind", [("lines", 64, 2560, 1021, 1056, 1), ("lines", 64, 1280, 1021, 1056, 0), ("large", 1, 600, 4090, 3850, 5),
                                                      ("large", 1, 16384, 1000, 1024, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_scale_and_nan(kernel, P, rows, N, K, behind, dtype):
    """X's scales from 1 to 247, a row of dY as far from 1 as X's is on the other side: sums of small integers.  Then a NaN scale and a NaN code,
    which reach their columns of their worker's gradient and nothing else."""
    import torch
    from paper_1901_04359_amd import binding as B
    each = rows // P
    if dtype == "f32" and kernel == "lines" and behind == 0:
        assert plan(dtype, P, rows, N, K, True)[0] == "lines"
    if dtype == "bf16":
        assert plan(dtype, P, rows, N, K, behind == 0 and N * K % 32 == 0)[0] == kernel
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows + K)
    per_row = torch.randint(1, 248, (rows, 1), device="cuda", generator=gen, dtype=torch.int32)
    per_row[0], per_row[1] = 1, 247
    d = torch.randint(-2, 3, (rows, N), device="cuda", generator=gen, dtype=torch.int32).double()
    dy = (d * torch.exp2(127.0 - per_row.double())).to(torch_type(dtype))
    x = torch.randint(-2, 3, (rows, K), device="cuda", generator=gen, dtype=torch.int64)
    nb = cdiv(K, 128)
    codes = torch.zeros(rows, nb * 128, dtype=torch.uint8, device="cuda")
    codes[:, :K] = torch.from_numpy(ref.encode(np.arange(-2.0, 3.0))).cuda()[x + 2]
    scales = per_row.to(torch.uint8).expand(rows, cdiv(nb, 4) * 4).contiguous()
    grads = torch.empty(P, behind + N * K, device="cuda")
    grad = grads[:, behind:].unflatten(1, (N, K))
    ws = B.alloc_weight_grad_workspace(rows, P, N, K)
    say(f"layer: weight_grad {dtype} P {P} rows {rows} {N}x{K}, every scale")
    B.gtopk_weight_grad(dy, codes, scales, None, grad, False, ws)
    want = [(d[w * each:(w + 1) * each].t().contiguous() @ x[w * each:(w + 1) * each].double()).float() for w in range(P)]
    for w in range(P):
        assert torch.equal(grad[w], want[w]), w
    last, t = P - 1, rows - 2
    scales[t, 2] = 255
    codes[t + 1, 7] = 0xFF
    B.gtopk_weight_grad(dy, codes, scales, None, grad, False, ws)
    gone = torch.zeros(K, dtype=torch.bool, device="cuda")
    gone[256:384], gone[7] = True, True
    for w in range(P):
        lost = torch.isnan(grad[w])
        assert torch.equal(lost, (gone & (w == last))[None, :].expand(N, K))
        assert torch.equal(grad[w][~lost], want[w][~lost])


# ---- bands of tiles, and long sums --------------------------------------------------------

@pytest.mark.parametrize("P,rows,N,K", [(1, 300, 300, 2336), (2, 800, 520, 1312), (3, 1100, 130, 4096)])
@pytest.mark.parametrize("dtype", TYPES)
def test_bands_of_tiles(P, rows, N, K, dtype):
    """More than four tiles across and several down, aligned rows, enough rows that writing does not bound the call: tiles in bands of four."""
    each = rows // P
    kernel, shares = plan(dtype, P, rows, N, K, True)
    assert each * PARTS[dtype] > 256 and cdiv(K, 256 if kernel == "wide" else 128) > 4 and N > 128 and kernel in ("small", "wide")
    begin = None if rows % P == 0 else [0, 100, 101, rows]
    check(P, rows, N, K, dtype, 0, 0, begin)


def test_a_sum_over_most_of_a_batch_past_32_bits():
    """Codes of more than 2^32 bytes, of which one worker has all but a few rows: its sum of half a million rows, in the first and the last columns."""
    import torch
    from paper_1901_04359_amd import binding as B
    rows, N, K, tail = 560_000, 12, 8192, 130
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    table = torch.from_numpy(ref.encode(np.arange(-2.0, 3.0))).cuda()
    codes = torch.empty(rows, K, dtype=torch.uint8, device="cuda")
    for at in range(0, rows, 70_000):
        codes[at:at + 70_000] = table[torch.randint(0, 5, (70_000, K), device="cuda", generator=gen, dtype=torch.uint8).int()]
    assert codes.numel() > 2 ** 32
    scales = torch.full((rows, 64), 127, dtype=torch.uint8, device="cuda")
    dy = torch.randint(-2, 3, (rows, N), device="cuda", generator=gen, dtype=torch.int32)
    begin = [0, 100, rows - tail, rows]
    plan_ = torch.tensor(begin, dtype=torch.int32, device="cuda")
    for dtype in TYPES:
        grad = torch.empty(3, N, K, device="cuda")
        say(f"layer: weight_grad {dtype} of a batch past 2^32 bytes")
        B.gtopk_weight_grad(dy.to(torch_type(dtype)), codes, scales, plan_, grad, False, B.alloc_weight_grad_workspace(rows, 3, N, K))
        for cols in (slice(0, 128), slice(4000, 4128), slice(K - 128, K)):
            x = codes[:, cols].contiguous().view(torch.float8_e4m3fn).double()
            for w in range(3):
                want = dy[begin[w]:begin[w + 1]].double().t().contiguous() @ x[begin[w]:begin[w + 1]]
                assert float(want.abs().max()) < 2 ** 24
                assert torch.equal(grad[w, :, cols].double(), want), (w, cols)
