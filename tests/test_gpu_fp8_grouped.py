"""8-bit products by expert as they are used: from operands quantised for them, on several streams, recorded with
boundaries that change, as a gradient; and what broken boundaries may not do."""
import pytest
import torch

from paper_2512_12949_amd import binding as ff

import grouped_util as u

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def _quantise(x, block=1, transpose=False):
    m, k = x.shape[::-1] if transpose else x.shape
    q = torch.empty((m, (k + 15) // 16 * 16), dtype=u.E4M3, device="cuda")
    s = torch.empty(((k + 127) // 128, (m + block - 1) // block), device="cuda")
    ff.ffuse_fp8_quantize(u.CODE[x.dtype], x, q, s, block_rows=block, transpose=transpose)
    return q, s


def _weights(W, block, transpose):
    laid = [_quantise(w, block, transpose) for w in W]
    return torch.stack([q.view(torch.uint8) for q, _ in laid]).view(u.E4M3), torch.stack([s for _, s in laid])


def _check(Y, A, sa, B, sb, block, t, what):
    """One group against its quantised operands in 64 bits.  fp32 sums: of a block's sixteen eights, the scales' product, the blocks;
    before them, in each eight, seven products that lose less than 2^-13 of the largest."""
    a, b = u.values64(A, sa, 1), u.values64(B, sb, block)
    want, err = a @ b.t(), (a.abs() @ b.abs().t()) * (32 + 2 * sa.shape[0]) * 2.0 ** -23
    for k in range(0, a.shape[1], 8):
        err += 7 * 2.0 ** -13 * (a[:, None, k:k + 8].abs() * b[None, :, k:k + 8].abs()).amax(dim=2)
    u.assert_within(Y, want, u.rounded(want, err, t), what)


@pytest.mark.parametrize("sizes", [[1, 0, 3], [40, 0, 129, 64], [300, 700]])
@pytest.mark.parametrize("K,N", [(136, 72), (520, 264)])
@pytest.mark.parametrize("t", (BF16, F16))
def test_a_step_by_expert(sizes, K, N, t):
    """The product and the gradient of its input, each from weights quantised in its own orientation; rows of no group stay."""
    gen, E, head, tail = torch.Generator().manual_seed(50), len(sizes), 2, 3
    R = sum(sizes) + head + tail
    X, dY, W = u.normal(gen, (R, K), 1.0, t), u.normal(gen, (R, N), 0.1, t), u.normal(gen, (E, K, N), K ** -0.5, t)
    off = u.offsets_of(sizes, head)
    Y, dX = torch.full((R, N), 7.0, dtype=t, device="cuda"), torch.full((R, K), 7.0, dtype=t, device="cuda")
    x, d, wt, w = _quantise(X), _quantise(dY), _weights(W, 128, True), _weights(W, 128, False)
    ff.ffuse_grouped_gemm_fp8(u.CODE[t], *x, *wt, off, Y)
    ff.ffuse_grouped_gemm_fp8(u.CODE[t], *d, *w, off, dX)
    torch.cuda.synchronize()
    at = head
    for e, n in enumerate(sizes):
        s = slice(at, at + n)
        at += n
        if not n:
            continue
        _check(Y[s], x[0][s], x[1][:, s], wt[0][e], wt[1][e], 128, t, f"Y, group {e}")
        _check(dX[s], d[0][s], d[1][:, s], w[0][e], w[1][e], 128, t, f"dX, group {e}")
        # against the unquantised operands: each is off by 2^-4 of itself at most, or by half the smallest number, 2^-10, times its block's
        # scale, which is at most the largest of the block / 224
        for got, a, b in ((Y[s], X[s], W[e]), (dX[s], dY[s], W[e].t())):
            a, b = a.double(), b.double()
            slack = (a.abs() @ b.abs()) * (2 * 2.0 ** -4 + 2.0 ** -8 + 2.0 ** -7) + a.abs().max() * b.abs().max() * a.shape[1] * 2 * 2.0 ** -16
            assert bool(((got.double() - a @ b).abs() <= slack).all())
    for out in (Y, dX):
        assert bool((out[:head] == 7).all()) and bool((out[R - tail:] == 7).all())


@pytest.mark.parametrize("R,N,block", [(6, 40, 128), (6, 40, 1), (12, 264, 1), (200, 264, 128), (200, 264, 1)])      # few rows stream, many use tiles
def test_boundaries_that_are_not_boundaries(R, N, block):
    """Decreasing and far-off boundaries: unspecified rows, but nothing outside the outputs is written, nor outside the operands read
    (their neighbours are NaN)."""
    gen, E, K, guard = torch.Generator().manual_seed(51), 6, 144, 4096
    A = torch.full(((R + 64) * K,), 0x7f, dtype=torch.uint8, device="cuda")
    A[32 * K:(32 + R) * K] = torch.randint(0, 0x70, (R * K,), generator=gen, dtype=torch.uint8).cuda()
    A = A[32 * K:(32 + R) * K].view(R, K).view(u.E4M3)
    B = torch.randint(0, 0x70, (E, N, K), generator=gen, dtype=torch.uint8).cuda().view(u.E4M3)
    sa, sb = torch.rand((2, R), generator=gen).cuda(), torch.rand((E, 2, (N + block - 1) // block), generator=gen).cuda()
    for values in ([5, -3, 100000, 2, R, 7, 12], [R] * 7, [-(2 ** 31)] * 3 + [2 ** 31 - 1] * 4, [0, R, 0, R, 0, R, 0], [R, 0, 0, 0, 0, 0, 0]):
        print("boundaries", R, N, block, values, flush=True)
        buf = torch.full((R * N + 2 * guard,), 3.0, dtype=BF16, device="cuda")
        ff.ffuse_grouped_gemm_fp8(ff.DT_BF16, A, sa, B, sb, torch.tensor(values, dtype=torch.int32, device="cuda"), buf[guard:guard + R * N].view(R, N))
        torch.cuda.synchronize()
        assert bool((buf[:guard] == 3).all()) and bool((buf[guard + R * N:] == 3).all()) and bool(torch.isfinite(buf).all())


def test_a_chain_whose_boundaries_are_none():
    """The chain by expert: output and workspace."""
    gen, K, N1, N2, R, E, guard = torch.Generator().manual_seed(52), 72, 136, 40, 200, 6, 4096
    X, W1, W2 = u.normal(gen, (R, K), 1.0, BF16), u.normal(gen, (E, K, N1), 0.1, BF16), u.normal(gen, (E, N1, N2), 0.1, BF16)
    nbytes = ff.ffuse_grouped_workspace_bytes(ff.DT_BF16, R, N1)
    for values in ([5, -3, 100000, 2, R, 7, 12], [R] * 7, [-(2 ** 31)] * 3 + [2 ** 31 - 1] * 4, [0, R, 0, R, 0, R, 0]):
        buf = torch.full((R * N2 + 2 * guard,), 3.0, dtype=BF16, device="cuda")
        ws = torch.full((nbytes + 2 * guard,), 9, dtype=torch.uint8, device="cuda")
        off = torch.tensor(values, dtype=torch.int32, device="cuda")
        ff.ffuse_grouped_ffn(ff.DT_BF16, X, W1, None, W2, off, ff.ACT_RELU, buf[guard:guard + R * N2].view(R, N2), ws[guard:guard + nbytes])
        torch.cuda.synchronize()
        assert bool((buf[:guard] == 3).all()) and bool((buf[guard + R * N2:] == 3).all())
        assert bool((ws[:guard] == 9).all()) and bool((ws[guard + nbytes:] == 9).all())


@pytest.mark.parametrize("R", (12, 300))
def test_recorded_with_new_boundaries_each_replay(R):
    """Quantised and multiplied in a graph; replays read the boundaries and rows they then find."""
    gen, K, N, E = torch.Generator().manual_seed(53), 136, 264, 5
    X, W = u.normal(gen, (R, K), 1.0, BF16), u.normal(gen, (E, K, N), K ** -0.5, BF16)
    w, off = _weights(W, 128, True), u.offsets_of([R // E] * E)
    q, s, Y = torch.empty((R, 144), dtype=u.E4M3, device="cuda"), torch.empty((2, R), device="cuda"), torch.empty((R, N), dtype=BF16, device="cuda")

    def step():
        ff.ffuse_fp8_quantize(ff.DT_BF16, X, q, s)
        ff.ffuse_grouped_gemm_fp8(ff.DT_BF16, q, s, *w, off, Y)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
    torch.cuda.synchronize()
    for sizes in ([R // E] * E, [0, R, 0, 0, 0], [1, 2, 3, 4, R - 10], [R // 2, 0, R // 4, 1, 0]):
        off.copy_(u.offsets_of(sizes))
        X.copy_(u.normal(gen, (R, K), 1.0, BF16))
        Y.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        replayed = Y.clone()
        torch.randn(1 << 20, device="cuda").sum()
        Y.fill_(7.0)
        step()
        torch.cuda.synchronize()
        assert torch.equal(replayed, Y), sizes
        at = 0
        for e, n in enumerate(sizes):
            if n:
                _check(Y[at:at + n], q[at:at + n], s[:, at:at + n], w[0][e], w[1][e], 128, BF16, f"{sizes}, group {e}")
            at += n
        assert bool((Y[at:] == 7).all())


def test_two_streams_at_once():
    gen, K, N = torch.Generator().manual_seed(54), 264, 520
    sizes = [[100, 0, 400, 37], [1, 0, 2, 1]]
    work = []
    for s in sizes:
        X, W = u.normal(gen, (sum(s), K), 1.0, BF16), u.normal(gen, (len(s), K, N), K ** -0.5, BF16)
        work.append((*_quantise(X), *_weights(W, 128, True), u.offsets_of(s)))
    alone = [torch.empty((sum(s), N), dtype=BF16, device="cuda") for s in sizes]
    out = [[torch.full((sum(s), N), float("nan"), dtype=BF16, device="cuda") for _ in range(20)] for s in sizes]
    for w, y in zip(work, alone):
        ff.ffuse_grouped_gemm_fp8(ff.DT_BF16, *w, y)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sizes]
    for i in range(20):
        for st, w, ys in zip(streams, work, out):
            with torch.cuda.stream(st):
                ff.ffuse_grouped_gemm_fp8(ff.DT_BF16, *w, ys[i])
    torch.cuda.synchronize()
    for ys, y in zip(out, alone):
        assert all(torch.equal(y, z) for z in ys)


@pytest.mark.parametrize("E", (512, 513, 1024))
def test_gated_products_of_many_small_groups(E):
    """On both sides of what the boundary tables leave room for; some experts have no rows."""
    gen, K, N = torch.Generator().manual_seed(55), 136, 72
    sizes = [(3 * i) % 4 if i % 3 else 0 for i in range(E)]
    R = sum(sizes)
    X, W, W3 = (torch.randn(s, device="cuda").to(BF16) for s in ((R, K), (E, K, N), (E, K, N)))
    Y = torch.empty((R, N), dtype=BF16, device="cuda")
    ff.ffuse_grouped_gemm(ff.DT_BF16, X, W / 8, W3 / 8, u.offsets_of(sizes), ff.ACT_SILU, Y)
    torch.cuda.synchronize()
    at = 0
    for e, n in enumerate(sizes):
        if n and (e % 29 == 1 or e > E - 3):
            u.assert_within(Y[at:at + n], *u.product64(X[at:at + n], W[e] / 8, W3[e] / 8, ff.ACT_SILU, BF16), f"group {e}")
        at += n
    assert bool(torch.isfinite(Y).all())
