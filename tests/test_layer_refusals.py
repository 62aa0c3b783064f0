"""Host-side checks of the layer calls: every bad argument becomes an error code, without touching a GPU."""
import ctypes

import numpy as np
import pytest

from paper_1901_04359_amd import binding as B
from tests import layer_reference as ref

FAKE = ctypes.c_void_p(0x10000)        # aligned, never dereferenced: every call below is rejected
ODD = ctypes.c_void_p(0x10004)         # aligned for four bytes
UNEVEN = ctypes.c_void_p(0x10001)
EINVAL, EALIGN, EWS, OK = B.GTOPK_EINVAL, B.GTOPK_EALIGN, B.GTOPK_EWORKSPACE, B.GTOPK_OK


def call(name, defaults):
    f = getattr(B.load(), name)

    def run(**kw):
        assert set(kw) <= set(defaults), kw
        return f(*{**defaults, **kw}.values())
    return run


def test_pack_rows():
    f = call("gtopk_pack_rows", dict(x=FAKE, dtype=0, rows=3, cols=130, stride=130, codes=FAKE, cs=256, scales=FAKE, ss=4, st=None))
    for kw in (dict(x=None), dict(codes=None), dict(scales=None), dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(rows=2**31),
               dict(cols=0), dict(cols=2**31), dict(stride=129), dict(cs=128), dict(cs=320), dict(ss=1), dict(ss=6)):
        assert f(**kw) == EINVAL, kw
    for kw in (dict(x=UNEVEN), dict(codes=ODD), dict(scales=UNEVEN), dict(x=UNEVEN, dtype=1)):
        assert f(**kw) == EALIGN, kw
    assert f(rows=0, x=None, codes=None, scales=None) == OK


def test_pack_tiles():
    f = call("gtopk_pack_tiles", dict(x=FAKE, dtype=0, rows=3, cols=130, stride=130, codes=FAKE, cs=256, scales=FAKE, ss=4,
                                      ct=FAKE, cts=128, sct=FAKE, scts=4, st=None))
    for kw in (dict(x=None), dict(codes=None), dict(scales=None), dict(ct=None), dict(sct=None), dict(dtype=3), dict(rows=-1),
               dict(cols=0), dict(stride=129), dict(cs=128), dict(cts=64), dict(cts=0), dict(ss=0), dict(scts=3),
               dict(codes=None, scales=None, ct=None, sct=None)):
        assert f(**kw) == EINVAL, kw
    for kw in (dict(x=UNEVEN), dict(codes=ODD), dict(ct=ODD), dict(sct=UNEVEN)):
        assert f(**kw) == EALIGN, kw
    assert f(rows=0, x=None) == OK


def test_unpack_and_activation_grad():
    f = call("gtopk_unpack", dict(codes=FAKE, cs=256, scales=FAKE, ss=4, rows=3, cols=130, act=0, out=FAKE, dtype=1, os=130, st=None))
    for kw in (dict(codes=None), dict(scales=None), dict(out=None), dict(cs=128), dict(ss=2), dict(rows=-1), dict(cols=0), dict(act=6),
               dict(act=-1), dict(dtype=9), dict(os=129)):
        assert f(**kw) == EINVAL, kw
    for kw in (dict(codes=ODD), dict(scales=UNEVEN), dict(out=UNEVEN)):
        assert f(**kw) == EALIGN, kw
    assert f(rows=0, codes=None, out=None) == OK
    f = call("gtopk_activation_grad", dict(codes=FAKE, cs=256, scales=FAKE, ss=4, rows=3, cols=130, act=0, dy=FAKE, dys=130, dx=FAKE,
                                           dxs=130, dtype=1, st=None))
    for kw in (dict(codes=None), dict(scales=None), dict(dy=None), dict(dx=None), dict(cs=255), dict(ss=0), dict(rows=-1), dict(cols=0),
               dict(act=6), dict(dtype=3), dict(dys=129), dict(dxs=129), dict(dxs=131)):       # the last: in place, at two strides
        assert f(**kw) == EINVAL, kw
    for kw in (dict(codes=ODD), dict(scales=UNEVEN), dict(dy=UNEVEN), dict(dx=UNEVEN)):
        assert f(**kw) == EALIGN, kw
    assert f(rows=0) == OK


def test_scaled_product():
    ws = B.gtopk_product_workspace_bytes(5, 7, 130)
    assert ws > 0 and B.gtopk_product_workspace_bytes(0, 7, 130) > 0
    for bad in ((-1, 7, 130), (5, 0, 130), (5, 7, 0), (2**31, 7, 130), (5, 2**31, 130), (5, 7, 2**31), (5, 7, 2**23 + 1), (32, 2**26 + 1, 8),
                (2**31 - 1, 1, 1), (2**19, 2**19, 1)):
        assert B.gtopk_product_workspace_bytes(*bad) == 0
    f = call("gtopk_scaled_product", dict(a=FAKE, acs=256, asc=FAKE, ass=4, b=FAKE, bcs=256, bsc=FAKE, bss=4, M=5, N=7, K=130,
                                          out=FAKE, dtype=0, os=7, ws=FAKE, wsb=ws, st=None))
    for kw in (dict(a=None), dict(asc=None), dict(b=None), dict(bsc=None), dict(out=None), dict(ws=None), dict(M=-1), dict(N=0), dict(K=0),
               dict(acs=128), dict(bcs=128), dict(acs=257), dict(ass=1), dict(bss=7), dict(dtype=3), dict(os=6), dict(acs=2**23 + 128),
               dict(bcs=2**23 + 128), dict(ass=2**23 + 4), dict(bss=2**23 + 4)):
        assert f(**kw) == EINVAL, kw
    for kw in (dict(a=ODD), dict(b=ODD), dict(asc=UNEVEN), dict(bsc=UNEVEN), dict(out=UNEVEN), dict(ws=ODD)):
        assert f(**kw) == EALIGN, kw
    assert f(wsb=ws - 1) == EWS
    assert f(M=0, a=None, out=None) == OK


def test_weight_grad():
    ws = B.gtopk_weight_grad_workspace_bytes(6, 3, 7, 130)
    assert ws > 0 and B.gtopk_weight_grad_workspace_bytes(0, 3, 7, 130) > 0
    for bad in ((-1, 3, 7, 130), (6, 0, 7, 130), (6, 32769, 7, 130), (6, 3, 0, 130), (6, 3, 7, 0), (2**31, 3, 7, 130)):
        assert B.gtopk_weight_grad_workspace_bytes(*bad) == 0
    f = call("gtopk_weight_grad", dict(dy=FAKE, dtype=1, dys=7, codes=FAKE, cs=256, scales=FAKE, ss=4, rows=6, begin=FAKE, P=3, N=7,
                                       K=130, grad=FAKE, gs=910, acc=0, ws=FAKE, wsb=ws, st=None))
    for kw in (dict(dy=None), dict(codes=None), dict(scales=None), dict(grad=None), dict(ws=None), dict(dtype=3), dict(dys=6), dict(cs=128),
               dict(ss=1), dict(rows=-1), dict(P=0), dict(P=32769), dict(N=0), dict(K=0), dict(gs=909), dict(begin=None, rows=7)):
        assert f(**kw) == EINVAL, kw
    for kw in (dict(dy=UNEVEN), dict(codes=ODD), dict(scales=UNEVEN), dict(begin=UNEVEN), dict(grad=UNEVEN), dict(ws=ODD)):
        assert f(**kw) == EALIGN, kw
    assert f(wsb=ws - 1) == EWS


def test_binding_refusals():
    import torch
    x, u = torch.zeros(4, 130), torch.zeros(4, 256, dtype=torch.uint8)
    for f in (lambda: B.gtopk_pack_rows(x, u, u), lambda: B.gtopk_pack_rows(x.double(), u, u), lambda: B.gtopk_pack_tiles(x, u, u),
              lambda: B.gtopk_unpack(u, u, "relu", x), lambda: B.gtopk_activation_grad(u, u, "relu", x, x),
              lambda: B.gtopk_scaled_product(u, u, u, u, 130, x, u),
              lambda: B.gtopk_weight_grad(x, u, u, None, torch.zeros(2, 130, 130), False, u)):
        with pytest.raises(TypeError):             # CPU tensors, and a type that no call takes
            f()
    with pytest.raises(ValueError):
        B._act_code("softmax")
    with pytest.raises(ValueError):
        B._packed(u, torch.zeros(4, 2, dtype=torch.uint8), 4, 130, torch, "")      # scales not in fours
    with pytest.raises(ValueError):
        B._packed(u, torch.zeros(4, 4, dtype=torch.uint8), 4, 257, torch, "")      # too few codes
    with pytest.raises(ValueError):
        B._packed(u, torch.zeros(3, 4, dtype=torch.uint8), 4, 130, torch, "")      # another number of rows
    with pytest.raises(ValueError):
        B._dense(x.t(), torch, "x")
    with pytest.raises(B.GtopkError):
        B.alloc_product_workspace(4, 0, 4)
    with pytest.raises(B.GtopkError):
        B.alloc_weight_grad_workspace(4, 0, 4, 4)


def test_reference_pack():
    """The reference itself, against the definition: the exponent is the smallest that will do, codes are nearest."""
    r = np.random.default_rng(3)
    for top in [448.0, 448.0 * (1 + 2.0**-23), 1.0, 1.75, 1.7500001, 2.0**-149, 3e38, *np.exp(r.uniform(-80, 80, 50))]:
        s = ref.exponent(float(top))
        assert top <= 448.0 * 2.0 ** (s - 127) and (s == 0 or top > 448.0 * 2.0 ** (s - 128))
    y = np.concatenate([r.uniform(-448, 448, 500), r.uniform(-0.02, 0.02, 500), [448.0, 464.0 - 16.0, 2.0**-10, -2.0**-10, 3 * 2.0**-10]])
    v = ref.CODE_VALUES[ref.encode(y)]
    finite = ref.CODE_VALUES[np.isfinite(ref.CODE_VALUES)]
    assert np.array_equal(np.abs(v - y), np.abs(finite[None, :] - y[:, None]).min(axis=1))
    assert list(ref.encode(np.array([2.0**-10, 3 * 2.0**-10, 17.0, 19.0]))) == [0, 2, 0x58, 0x5A]     # ties to the even code
