"""The rules by which a weight gradient takes its tiles, as the GPU tests write them out: both sides of each line, and the shares of the rows
against the workspace that the library asks for."""
import random

from paper_1901_04359_amd import binding as B
from tests.test_gpu_layer_plans import plan


def test_the_rule_for_lines():
    """Both sides of each of its lines."""
    for dtype, P, each, N, K, aligned, lines in (
            ("bf16", 16, 64, 4096, 9216, False, True), ("bf16", 8, 64, 1000, 4096, True, False), ("bf16", 16, 256, 2048, 2048, True, True),
            ("bf16", 16, 257, 2048, 2048, True, False), ("bf16", 16, 128, 2048, 2048, False, True), ("bf16", 16, 129, 2048, 2048, False, False),
            ("bf16", 512, 64, 512, 512, False, False), ("f32", 16, 85, 2048, 2048, True, True), ("f32", 16, 86, 2048, 2048, True, False),
            ("f32", 16, 21, 4096, 4096, False, True), ("f16", 16, 33, 4096, 4096, False, False), ("f16", 16, 32, 4096, 4064, False, False),
            ("bf16", 16, 64, 4096, 9217, True, False)):
        assert (plan(dtype, P, P * each, N, K, aligned)[0] == "lines") == lines


def test_the_rule_for_large_tiles():
    """Both sides of each of its lines, by sizes whose times stand beside it."""
    for P, rows, N, K, large in ((1, 512, 4096, 4096, True), (1, 511, 4096, 4096, False), (1, 2048, 5120, 5120, True), (1, 2048, 4096, 5120, False),
                                 (1, 2048, 4096, 9216, False), (1, 8192, 8192, 8192, True), (1, 16384, 1024, 1024, True), (1, 8192, 1024, 1024, False),
                                 (1, 4096, 2048, 2048, True), (1, 2048, 2048, 2048, False), (1, 4096, 2048, 4096, True), (1, 2048, 2048, 4096, False)):
        assert (plan("bf16", P, rows, N, K, True)[0] == "large") == large


def test_shares_are_those_of_the_workspace():
    """A share of every worker's gradient each, in fp32 and padded to fours: the most that any type needs."""
    r = random.Random(5)
    for _ in range(3000):
        P, N, K = 2 ** r.randint(0, 6), int(2 ** r.uniform(0, 13)), int(2 ** r.uniform(0, 13))
        rows = P * int(2 ** r.uniform(0, 15))
        most = max(plan(dtype, P, rows, N, K, False)[1] for dtype in ("f32", "bf16"))
        want = 256 + (4 * most * P * -(-N * K // 4) * 4 if most > 1 else 0)
        assert B.gtopk_weight_grad_workspace_bytes(rows, P, N, K) == want, (P, rows, N, K)
