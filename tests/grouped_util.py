"""Plain forms in 64 bits of the products grouped by expert and of the 8-bit products, with the error that the
library's arithmetic may have: one rounding of the result (half a step of its type), and fp32 sums, each of whose n
additions is off by at most 2^-23 of the sum of the magnitudes (the matrix pipe may truncate)."""
import math

import torch

from paper_2512_12949_amd import binding as ff

CODE = {torch.bfloat16: ff.DT_BF16, torch.float16: ff.DT_F16}
E4M3 = torch.float8_e4m3fn


def half_step(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    """Half the distance of the smallest numbers of a type."""
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def offsets_of(sizes, first=0):
    return torch.tensor([first + sum(sizes[:i]) for i in range(len(sizes) + 1)], dtype=torch.int32, device="cuda")


def normal(gen, shape, std, t):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * std).to(t).cuda()


def act64(act, x):
    if act == ff.ACT_RELU:
        return torch.clamp(x, min=0)
    if act == ff.ACT_GELU_TANH:
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    return x / (1 + torch.exp(-x)) if act == ff.ACT_SILU else x


def mm(a, b):
    """a @ b and the error of fp32 sums of the same products."""
    a, b = a.double(), b.double()
    return a @ b, (a.abs() @ b.abs()) * (a.shape[1] + 8) * 2.0 ** -23


def rounded(y, err, t):
    """What the error becomes when y +- err is rounded to type t."""
    return err + (y.abs() + err) * half_step(t) + tiny(t)


def product64(x, w, w3, act, t):
    """One group's product and its error.  The activations' slopes are at most 1.13, their own arithmetic (exp and
    reciprocal of the hardware) is good to 4e-6 of the larger of value and argument."""
    g, eg = mm(x, w)
    y = act64(act, g)
    e = eg if act in (ff.ACT_IDENTITY, ff.ACT_RELU) else 1.13 * eg + 4e-6 * torch.maximum(y.abs(), g.abs())
    if w3 is not None:
        u, eu = mm(x, w3)
        e = e * u.abs() + y.abs() * eu + e * eu + (y * u).abs() * 2.0 ** -23
        y = y * u
    return y, rounded(y, e, t)


def assert_within(got, want, err, what):
    got = got.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = ((got - want).abs() - err).max().item() if got.numel() else 0.0
    worst = ((got - want).abs() / err.clamp(min=1e-300)).max().item() if got.numel() else 0.0
    assert over <= 0, f"{what}: {worst:.3g} times the error it may have"


def scale64(top):
    """The scale of a block whose largest finite magnitude is `top`."""
    if top == 0:
        return 1.0
    m, e = math.frexp(top)     # top = m 2^e, m in [0.5, 1)
    return 2.0 ** max(-126, e - 9 if m <= 0.875 else e - 8)


def values64(q, scale, rows):
    """What e4m3 numbers and their scales [blocks of 128][blocks of rows] stand for."""
    s = scale.double().t().repeat_interleave(rows, 0)[: q.shape[0]].repeat_interleave(128, 1)[:, : q.shape[1]]
    return q.double() * s
