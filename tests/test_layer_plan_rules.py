"""The rules by which a weight gradient takes its tiles, as the GPU tests write them out: both sides of each line, and the shares of the rows
against the workspace that the library asks for."""
import random

from paper_1901_04359_amd import binding as B
from tests.test_gpu_layer_plans import plan


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
