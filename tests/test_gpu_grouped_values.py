"""NaN and infinities through the products and the chain by expert: where the definition has them, and nowhere else."""
import pytest
import torch

from paper_2512_12949_amd import binding as ff

import grouped_util as u

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
ACTS = (ff.ACT_IDENTITY, ff.ACT_RELU, ff.ACT_GELU_TANH, ff.ACT_SILU)
NAN, INF = float("nan"), float("inf")


def _same(got, want, what):
    """NaN and infinities where `want` has them (finite values have tests of their own)."""
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN"
    assert torch.equal(got.where(torch.isinf(want), torch.zeros_like(got)), want.where(torch.isinf(want), torch.zeros_like(want))), f"{what}: infinities"
    assert torch.equal(torch.isinf(got), torch.isinf(want)), f"{what}: infinities"


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gated", (False, True))
@pytest.mark.parametrize("t", (BF16, F16))
@pytest.mark.parametrize("sizes", [[3, 1], [40, 0, 65], [700, 20]])
def test_not_a_number_and_infinities(act, gated, t, sizes):
    gen, K, N, N2 = torch.Generator().manual_seed(40), 136, 264, 72
    R, E = sum(sizes), len(sizes)
    X, W, W2 = u.normal(gen, (R, K), 1.0, t), u.normal(gen, (E, K, N), K ** -0.5, t), u.normal(gen, (E, N, N2), N ** -0.5, t)
    W3 = u.normal(gen, (E, K, N), K ** -0.5, t) if gated else None
    X[0, 5] = NAN
    X[1, 7], X[2, 9] = INF, -INF
    X[R - 1, 3], X[R - 1, 4] = INF, INF       # of both signs in some columns: NaN there
    W[0, 11, 100], W[E - 1, K - 1, N - 1] = NAN, INF
    if gated:
        W3[0, 2, 33], W3[E - 1, 8, 40] = NAN, -INF
    off, Y, Z = u.offsets_of(sizes), torch.empty((R, N), dtype=t, device="cuda"), torch.empty((R, N2), dtype=t, device="cuda")
    ws = torch.empty(ff.ffuse_grouped_workspace_bytes(u.CODE[t], R, N), dtype=torch.uint8, device="cuda")
    ff.ffuse_grouped_gemm(u.CODE[t], X, W, W3, off, act, Y)
    ff.ffuse_grouped_ffn(u.CODE[t], X, W, W3, W2, off, act, Z, ws)
    torch.cuda.synchronize()
    a = 0
    for e, n in enumerate(sizes):
        s = slice(a, a + n)
        a += n
        x = X[s].double()
        h = u.act64(act, x @ W[e].double())
        if gated:
            h = h * (x @ W3[e].double())
        assert bool(torch.isnan(h).any()) or not n
        _same(Y[s], h, f"product, group {e}")
        _same(Z[s], h @ W2[e].double(), f"chain, group {e}")


@pytest.mark.parametrize("t", (BF16, F16))
def test_relu_at_and_around_zero(t):
    """max(x, 0) to the bit: the smallest numbers of either sign, zeros, the largest."""
    info = torch.finfo(t)
    small = info.smallest_normal * info.eps
    v = torch.tensor([0.0, -0.0, small, -small, info.smallest_normal, -info.smallest_normal, 1.0, -1.0, info.max, info.min, INF, -INF, NAN, 3.0, -3.0, 0.5],
                     dtype=torch.float64).to(t)
    X = torch.zeros((16, 16), dtype=t)
    X[:, 0] = 1.0
    W = torch.zeros((1, 16, 16), dtype=t)
    W[0, 0] = v
    Y = torch.empty((16, 16), dtype=t, device="cuda")
    ff.ffuse_grouped_gemm(u.CODE[t], X.cuda(), W.cuda(), None, u.offsets_of([16]), ff.ACT_RELU, Y)
    want = torch.clamp(v, min=0).expand(16, 16)
    # (a subnormal may come out of the matrix instruction as zero)
    tiny = (want > 0) & (want < info.smallest_normal)
    got = Y.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[~tiny & ~torch.isnan(want)], want[~tiny & ~torch.isnan(want)])
