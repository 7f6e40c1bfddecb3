"""What the products by expert and the 8-bit products refuse, before any device work."""
import ctypes

import pytest
import torch

from paper_2512_12949_amd import binding as ff

P, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)   # never dereferenced: validation fails first
NULL, SHAPE, ALIGN, ACT = -1, -2, -3, -4


def _grouped(name, **kw):
    """One call with good arguments but for kw."""
    v = dict(dtype=0, a=P, w=P, w3=None, off=P, act=0, R=4, E=2, K=16, N=16, y=P)
    v.update(kw)
    f = getattr(ff.lib(), name)
    if name == "ffuse_grouped_gemm":
        return f(v["dtype"], v["a"], v["w"], v["w3"], v["off"], v["act"], v["R"], v["E"], v["K"], v["N"], v["y"], None)
    return f(v["dtype"], v["a"], v["w"], v["off"], v["R"], v["E"], v["K"], v["N"], v["y"], None)


@pytest.mark.parametrize("name", ("ffuse_grouped_gemm", "ffuse_grouped_gemm_dx", "ffuse_grouped_gemm_dw"))
def test_grouped_products(name):
    for kw, want in ((dict(a=None), NULL), (dict(w=None), NULL), (dict(off=None), NULL), (dict(y=None), NULL),
                     (dict(dtype=2), ACT), (dict(dtype=-1), ACT), (dict(R=-1), SHAPE), (dict(R=1 << 31), SHAPE), (dict(E=0), SHAPE), (dict(E=1025), SHAPE),
                     (dict(K=0), SHAPE), (dict(K=12), SHAPE), (dict(N=4), SHAPE), (dict(N=20), SHAPE), (dict(K=1 << 21), SHAPE),
                     (dict(K=1 << 16, N=1 << 14), SHAPE), (dict(a=ODD), ALIGN), (dict(w=ODD), ALIGN), (dict(y=ODD), ALIGN),
                     (dict(off=ctypes.c_void_p(0x1002)), ALIGN)):
        assert _grouped(name, **kw) == want, (name, kw)
    if name == "ffuse_grouped_gemm":
        assert _grouped(name, act=4) == ACT and _grouped(name, act=-1) == ACT and _grouped(name, w3=ODD) == ALIGN
    if name == "ffuse_grouped_gemm_dw":
        assert _grouped(name, E=1024, K=16384, N=16384) == SHAPE      # more blocks than a launch has threads for


def test_grouped_chain():
    f = ff.lib().ffuse_grouped_ffn
    good = [0, P, P, P, P, P, 3, 4, 2, 16, 24, 32, P, P, 4 * 24 * 2, None]
    names = ["dtype", "X", "W1", "W3", "W2", "off", "act", "R", "E", "K", "N1", "N2", "Y", "ws", "bytes"]
    for key, value, want in (("X", None, NULL), ("W1", None, NULL), ("W2", None, NULL), ("off", None, NULL), ("Y", None, NULL), ("dtype", 2, ACT),
                             ("act", 9, ACT), ("E", 0, SHAPE), ("N1", 20, SHAPE), ("N2", 4, SHAPE), ("K", 0, SHAPE), ("W3", ODD, ALIGN), ("W2", ODD, ALIGN)):
        args = list(good)
        args[names.index(key)] = value
        assert f(*args) == want, key
    assert ff.ffuse_grouped_workspace_bytes(ff.DT_BF16, 100, 264) == 52992      # 2 * 100 * 264 up to a multiple of 256
    assert ff.ffuse_grouped_workspace_bytes(ff.DT_F32, 100, 264) == 0 and ff.ffuse_grouped_workspace_bytes(ff.DT_BF16, 100, 12) == 0
    assert ff.ffuse_grouped_workspace_bytes(ff.DT_BF16, 0, 264) == 0


def test_fp8():
    q = ff.lib().ffuse_fp8_quantize
    for args, want in (((0, None, 4, 16, 1, 0, P, P), NULL), ((0, P, 4, 16, 1, 0, None, P), NULL), ((0, P, 4, 16, 1, 0, P, None), NULL),
                       ((2, P, 4, 16, 1, 0, P, P), ACT), ((0, P, 4, 16, 64, 0, P, P), SHAPE), ((0, P, 4, 12, 1, 0, P, P), SHAPE), ((0, P, -1, 16, 1, 0, P, P), SHAPE),
                       ((0, P, 4, 1 << 21, 1, 0, P, P), SHAPE), ((0, ODD, 4, 16, 1, 0, P, P), ALIGN), ((0, P, 4, 16, 1, 0, ODD, P), ALIGN),
                       ((0, P, 4, 16, 1, 0, P, ctypes.c_void_p(0x1002)), ALIGN)):
        assert q(*args, None) == want, args
    g = ff.lib().ffuse_gemm_fp8
    for args, want in (((0, None, P, P, P, 1, 4, 16, 8, P), NULL), ((0, P, None, P, P, 1, 4, 16, 8, P), NULL), ((0, P, P, None, P, 1, 4, 16, 8, P), NULL),
                       ((0, P, P, P, None, 1, 4, 16, 8, P), NULL), ((0, P, P, P, P, 1, 4, 16, 8, None), NULL), ((2, P, P, P, P, 1, 4, 16, 8, P), ACT),
                       ((0, P, P, P, P, 2, 4, 16, 8, P), SHAPE), ((0, P, P, P, P, 1, 4, 24, 8, P), SHAPE), ((0, P, P, P, P, 1, 4, 16, 12, P), SHAPE),
                       ((0, P, P, P, P, 1, -4, 16, 8, P), SHAPE), ((0, ODD, P, P, P, 1, 4, 16, 8, P), ALIGN), ((0, P, P, ODD, P, 1, 4, 16, 8, P), ALIGN),
                       ((0, P, P, P, P, 1, 4, 16, 8, ODD), ALIGN), ((0, P, ctypes.c_void_p(0x1002), P, P, 1, 4, 16, 8, P), ALIGN)):
        assert g(*args, None) == want, args
    assert ff.lib().ffuse_grouped_gemm_fp8(0, P, P, P, P, 1, None, 4, 2, 16, 8, P, None) == NULL


def test_the_binding_checks_the_tensors():
    """Shape, type, contiguity and device: an address alone says none of them."""
    z = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t)  # noqa: E731
    off, e4m3 = torch.zeros(3, dtype=torch.int32), torch.float8_e4m3fn
    X, W, Y = z(4, 16), z(2, 16, 24), z(4, 24)
    call = ff.ffuse_grouped_gemm
    for bad in ((0, z(4, 8), W, None, off, 0, Y), (0, X, W, None, off[:2], 0, Y), (0, X, W, None, off.long(), 0, Y), (0, X, W, None, off, 0, z(4, 16)),
                (0, X, W, z(2, 16, 16), off, 0, Y), (1, X, W, None, off, 0, Y), (0, z(16, 4).t(), W, None, off, 0, Y), (2, X, W, None, off, 0, Y),
                (0, z(4), W, None, off, 0, Y), (0, X, z(16, 24), None, off, 0, Y)):
        with pytest.raises(ValueError):
            call(*bad)
    with pytest.raises(ValueError, match="current device"):      # on the CPU
        call(0, X, W, None, off, 0, Y)
    with pytest.raises(ValueError):
        ff.ffuse_grouped_gemm_dx(0, Y, W, off, z(4, 24))
    with pytest.raises(ValueError):
        ff.ffuse_grouped_gemm_dw(0, X, Y, off, z(2, 24, 16))
    with pytest.raises(ValueError):
        ff.ffuse_grouped_ffn(0, X, W, None, z(2, 16, 24), off, 0, Y, None)
    q, s = z(4, 32, t=e4m3), z(1, 4, t=torch.float32)
    with pytest.raises(ValueError):
        ff.ffuse_fp8_quantize(0, z(4, 24), z(4, 24, t=e4m3), s)             # rows of Q are padded to 16
    with pytest.raises(ValueError):
        ff.ffuse_fp8_quantize(0, z(4, 24), q, s.t())
    with pytest.raises(ValueError, match="scales of B"):
        ff.ffuse_gemm_fp8(0, q, s, z(8, 32, t=e4m3), z(1, 2, t=torch.float32), z(4, 8))
    with pytest.raises(ValueError):
        ff.ffuse_gemm_fp8(0, q, z(4, 1, t=torch.float32), z(8, 32, t=e4m3), z(1, 1, t=torch.float32), z(4, 8))
    with pytest.raises(ValueError):
        ff.ffuse_grouped_gemm_fp8(0, q, s, z(8, 32, t=e4m3), z(1, 1, t=torch.float32), off, z(4, 8))
