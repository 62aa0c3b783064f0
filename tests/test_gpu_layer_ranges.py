"""The layer calls at the ends of their ranges: values that fp32 cannot hold, the tails of the activation functions, scales from
the smallest on, and the sizes at which a weight gradient takes its large tiles or bands of tiles.

Tolerances are derived beside the tests.  u = 2^-24 is half a step of fp32."""
import math

import numpy as np
import pytest

from tests import layer_reference as ref
from tests.gpu_harness import say
from tests.test_gpu_layer import TYPES, half_step, packed_on_gpu, torch_type

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
