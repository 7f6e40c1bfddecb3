"""Products grouped by expert against the definition in 64 bits: ragged and empty groups, sizes on both sides of
every tile, rows of no group, neighbours full of NaN, tensors past 2^32 bytes, streams and graphs."""
import pytest
import torch

from paper_2512_12949_amd import binding as ff

import gpu_util as gu
import grouped_util as u

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
ACTS = (ff.ACT_IDENTITY, ff.ACT_RELU, ff.ACT_GELU_TANH, ff.ACT_SILU)
SIZES = {
    "one_row": [1],
    "first_and_last_empty": [0, 1, 0, 3, 0],
    "around_tiles": [1, 15, 16, 17, 31, 32, 33, 0, 63, 64, 65, 127, 128, 129, 255, 256, 257],
    "one_of_many": [0] * 70 + [40] + [0] * 70,
    "long": [700, 5, 1300],
    "many": [(7 * i) % 23 for i in range(150)],
}


def _spans(sizes, first=0):
    a = first
    for e, n in enumerate(sizes):
        yield e, slice(a, a + n)
        a += n


def _run_forward(sizes, K, N, t, act, gated, seed, head=0, tail=0):
    gen = torch.Generator().manual_seed(seed)
    R, E = sum(sizes) + head + tail, len(sizes)
    X, W = u.normal(gen, (R, K), 1.0, t), u.normal(gen, (E, K, N), K ** -0.5, t)
    W3 = u.normal(gen, (E, K, N), K ** -0.5, t) if gated else None
    X[:head] = float("nan")
    X[R - tail:] = float("nan")
    Y = torch.full((R, N), 7.0, dtype=t, device="cuda")
    off = u.offsets_of(sizes, head)
    print("forward", sizes[:4], len(sizes), K, N, t, act, gated, flush=True)
    ff.ffuse_grouped_gemm(u.CODE[t], X, W, W3, off, act, Y)
    torch.cuda.synchronize()
    for e, s in _spans(sizes, head):
        want, err = u.product64(X[s], W[e], None if W3 is None else W3[e], act, t)
        u.assert_within(Y[s], want, err, f"group {e} of {len(sizes)}, {sizes[e]} rows")
    assert bool((Y[:head] == 7).all()) and bool((Y[R - tail:] == 7).all() if tail else True)


@pytest.mark.parametrize("kind", SIZES)
@pytest.mark.parametrize("K,N", [(8, 8), (72, 24), (136, 264), (1000, 72), (256, 1032)])
def test_forward_sizes(kind, K, N):
    _run_forward(SIZES[kind], K, N, BF16, ff.ACT_IDENTITY, False, 1)
    _run_forward(SIZES[kind], K, N, F16, ff.ACT_SILU, True, 2)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gated", (False, True))
@pytest.mark.parametrize("t", (BF16, F16))
def test_forward_epilogues(act, gated, t):
    _run_forward([3, 0, 150, 33], 264, 136, t, act, gated, 3, head=5, tail=9)
    _run_forward([530, 290], 136, 520, t, act, gated, 4, head=1, tail=2)


@pytest.mark.parametrize("kind", SIZES)
@pytest.mark.parametrize("K,N", [(8, 8), (24, 72), (264, 136), (72, 1000), (1032, 256)])
@pytest.mark.parametrize("t", (BF16, F16))
def test_input_gradient(kind, K, N, t):
    gen, sizes, head, tail = torch.Generator().manual_seed(5), SIZES[kind], 3, 4
    R, E = sum(sizes) + head + tail, len(sizes)
    dY, W = u.normal(gen, (R, N), 0.1, t), u.normal(gen, (E, K, N), K ** -0.5, t)
    dY[:head] = float("nan")
    dY[R - tail:] = float("nan")
    dX = torch.full((R, K), 7.0, dtype=t, device="cuda")
    print("input", kind, K, N, t, flush=True)
    ff.ffuse_grouped_gemm_dx(u.CODE[t], dY, W, u.offsets_of(sizes, head), dX)
    torch.cuda.synchronize()
    for e, s in _spans(sizes, head):
        want, err = u.mm(dY[s], W[e].t())
        u.assert_within(dX[s], want, u.rounded(want, err, t), f"dX, group {e}")
    assert bool((dX[:head] == 7).all()) and bool((dX[R - tail:] == 7).all())


@pytest.mark.parametrize("kind", SIZES)
@pytest.mark.parametrize("K,N", [(8, 8), (24, 72), (264, 136), (72, 1000), (520, 264)])
@pytest.mark.parametrize("t", (BF16, F16))
def test_weight_gradient(kind, K, N, t):
    gen, sizes, head, tail = torch.Generator().manual_seed(6), SIZES[kind], 3, 4
    R, E = sum(sizes) + head + tail, len(sizes)
    X, dY = u.normal(gen, (R, K), 1.0, t), u.normal(gen, (R, N), 0.1, t)
    for x in (X, dY):
        x[:head] = float("nan")
        x[R - tail:] = float("nan")
    dW = torch.full((E, K, N), 7.0, dtype=t, device="cuda")
    print("weights", kind, K, N, t, flush=True)
    ff.ffuse_grouped_gemm_dw(u.CODE[t], X, dY, u.offsets_of(sizes, head), dW)
    torch.cuda.synchronize()
    for e, s in _spans(sizes, head):
        want, err = u.mm(X[s].t(), dY[s])
        if s.start == s.stop:
            assert bool((dW[e] == 0).all()), f"dW, empty group {e}"
        else:
            u.assert_within(dW[e], want, u.rounded(want, err, t), f"dW, group {e}")


def test_a_group_of_nan_stays_its_own():
    """NaN and infinities of one group's rows, gradients and weights reach no other group's results."""
    gen, sizes, K, N = torch.Generator().manual_seed(7), [37, 90, 65], 136, 72
    R = sum(sizes)
    X, W, dY = u.normal(gen, (R, K), 1.0, BF16), u.normal(gen, (3, K, N), 0.1, BF16), u.normal(gen, (R, N), 1.0, BF16)
    mid = slice(37, 127)
    X[mid], dY[mid], W[1] = float("nan"), float("inf"), float("nan")
    Y, dX, dW = torch.empty(R, N, dtype=BF16, device="cuda"), torch.empty(R, K, dtype=BF16, device="cuda"), torch.empty_like(W)
    off = u.offsets_of(sizes)
    ff.ffuse_grouped_gemm(ff.DT_BF16, X, W, None, off, ff.ACT_IDENTITY, Y)
    ff.ffuse_grouped_gemm_dx(ff.DT_BF16, dY, W, off, dX)
    ff.ffuse_grouped_gemm_dw(ff.DT_BF16, X, dY, off, dW)
    torch.cuda.synchronize()
    for out in (Y, dX):
        assert bool(torch.isfinite(out[:37]).all()) and bool(torch.isfinite(out[127:]).all()) and bool(torch.isnan(out[mid]).all())
    assert bool(torch.isfinite(dW[0]).all()) and bool(torch.isfinite(dW[2]).all()) and bool(torch.isnan(dW[1]).all())


def test_boundaries_that_are_not_boundaries_stay_inside_the_tensors():
    """Decreasing and far-off boundaries: unspecified rows, but nothing outside the outputs is written."""
    gen, K, N, R, E = torch.Generator().manual_seed(8), 72, 40, 200, 6
    X, W, dY = u.normal(gen, (R, K), 1.0, BF16), u.normal(gen, (E, K, N), 0.1, BF16), u.normal(gen, (R, N), 1.0, BF16)
    guard = 4096
    for values in ([5, -3, 100000, 2, R, 7, 12], [R] * 7, [-(2 ** 31)] * 3 + [2 ** 31 - 1] * 4, [0, R, 0, R, 0, R, 0]):
        off = torch.tensor(values, dtype=torch.int32, device="cuda")
        for call, shape in ((lambda y: ff.ffuse_grouped_gemm(ff.DT_BF16, X, W, None, off, ff.ACT_RELU, y), (R, N)),
                            (lambda y: ff.ffuse_grouped_gemm_dx(ff.DT_BF16, dY, W, off, y), (R, K)),
                            (lambda y: ff.ffuse_grouped_gemm_dw(ff.DT_BF16, X, dY, off, y), (E, K, N))):
            n = torch.Size(shape).numel()
            buf = torch.full((n + 2 * guard,), 3.0, dtype=BF16, device="cuda")
            call(buf[guard:guard + n].view(shape))
            torch.cuda.synchronize()
            assert bool((buf[:guard] == 3).all()) and bool((buf[guard + n:] == 3).all())


def test_no_rows():
    X, W, off = torch.empty((0, 64), dtype=BF16, device="cuda"), torch.ones((2, 64, 32), dtype=BF16, device="cuda"), u.offsets_of([0, 0])
    Y = torch.empty((0, 32), dtype=BF16, device="cuda")
    ff.ffuse_grouped_gemm(ff.DT_BF16, X, W, None, off, ff.ACT_RELU, Y)
    ff.ffuse_grouped_gemm_dx(ff.DT_BF16, Y, W, off, X)
    ff.ffuse_grouped_ffn(ff.DT_BF16, X, W, None, torch.ones((2, 32, 64), dtype=BF16, device="cuda"), off, ff.ACT_RELU, X, None)
    dW = torch.ones_like(W)
    ff.ffuse_grouped_gemm_dw(ff.DT_BF16, X, Y, off, dW)
    torch.cuda.synchronize()
    assert bool((dW == 0).all())


def test_gradients_agree_with_differences():
    """The product is linear in X and in W: its difference along a direction is the product of the direction, and has
    to be what the gradients say."""
    gen, sizes, K, N = torch.Generator().manual_seed(9), [100, 0, 57, 300], 200, 136
    R, E = sum(sizes), len(sizes)
    X, V, W, U = (u.normal(gen, s, 1.0, F16) for s in ((R, K), (R, K), (E, K, N), (E, K, N)))
    X, V, W, U = ((x / 8) for x in (X, V, W, U))
    dY, off = u.normal(gen, (R, N), 1.0, F16), u.offsets_of(sizes)
    out = lambda *s: torch.empty(s, dtype=F16, device="cuda")  # noqa: E731
    y = [out(R, N) for _ in range(4)]
    for Y, x, w in zip(y, (X + V, X - V, X, X), (W, W, W + U, W - U)):
        ff.ffuse_grouped_gemm(ff.DT_F16, x, w, None, off, ff.ACT_IDENTITY, Y)
    dX, dW = out(R, K), out(E, K, N)
    ff.ffuse_grouped_gemm_dx(ff.DT_F16, dY, W, off, dX)
    ff.ffuse_grouped_gemm_dw(ff.DT_F16, X, dY, off, dW)
    torch.cuda.synchronize()
    # Every rounding to fp16 is independent and off by 2^-11 at most: the outputs', the gradients', X +- V's and W +- U's
    # own.  Four standard deviations of such sums, each rounding taken at its bound.
    for (up, down), g, v in (((y[0], y[1]), dX, V), ((y[2], y[3]), dW, U)):
        diff = (dY.double() * (up.double() - down.double()) / 2).sum().item()
        said = (g.double() * v.double()).sum().item()
        noise = 2.0 ** -11 * ((dY.double() * torch.maximum(up.abs(), down.abs()).double()).norm().item() + (g.double() * v.double()).norm().item()
                              + (g.double() * (X.abs() + V.abs() if g is dX else W.abs() + U.abs()).double()).norm().item())
        assert abs(diff - said) <= 4 * noise, (diff, said, noise)


@pytest.mark.parametrize("t,act,gated", [(BF16, ff.ACT_SILU, True), (F16, ff.ACT_GELU_TANH, False)])
@pytest.mark.parametrize("sizes", [[1], [2, 0, 1, 0, 0, 3], [40, 200, 0, 129], [300, 513]])
def test_chain(t, act, gated, sizes):
    gen, K, N1, N2 = torch.Generator().manual_seed(10), 200, 328, 136
    R, E = sum(sizes) + 3, len(sizes)
    X, W1, W2 = u.normal(gen, (R, K), 1.0, t), u.normal(gen, (E, K, N1), K ** -0.5, t), u.normal(gen, (E, N1, N2), N1 ** -0.5, t)
    W3 = u.normal(gen, (E, K, N1), K ** -0.5, t) if gated else None
    off, Y = u.offsets_of(sizes), torch.full((R, N2), 7.0, dtype=t, device="cuda")
    ws = torch.empty(ff.ffuse_grouped_workspace_bytes(u.CODE[t], R, N1), dtype=torch.uint8, device="cuda")
    ff.ffuse_grouped_ffn(u.CODE[t], X, W1, W3, W2, off, act, Y, ws)
    torch.cuda.synchronize()
    for e, s in _spans(sizes):
        h, eh = u.product64(X[s], W1[e], None if W3 is None else W3[e], act, t)
        want, err = u.mm(h, W2[e])
        u.assert_within(Y[s], want, u.rounded(want, err + eh @ W2[e].double().abs(), t), f"chain, group {e}")
    assert bool((Y[R - 3:] == 7).all())


def test_rows_and_weights_past_32_bits():
    """X and Y of 5 and 3 GiB, 6 GiB of weights: the last rows and the last expert."""
    K, N, E, R = 8192, 4104, 96, 330000
    X = torch.zeros((R, K), dtype=BF16, device="cuda")
    W = torch.zeros((E, K, N), dtype=BF16, device="cuda")
    gen = torch.Generator().manual_seed(11)
    n = 70
    X[R - n:], W[E - 1] = u.normal(gen, (n, K), 1.0, BF16), u.normal(gen, (K, N), K ** -0.5, BF16)
    sizes = [0] * (E - 2) + [R - n, n]
    off, Y = u.offsets_of(sizes), torch.full((R, N), 7.0, dtype=BF16, device="cuda")
    ff.ffuse_grouped_gemm(ff.DT_BF16, X, W, None, off, ff.ACT_IDENTITY, Y)
    want, err = u.mm(X[R - n:], W[E - 1])
    u.assert_within(Y[R - n:], want, u.rounded(want, err, BF16), "last group")
    assert bool((Y[: R - n] == 0).all())
    dX = torch.full_like(X, 7.0)
    ff.ffuse_grouped_gemm_dx(ff.DT_BF16, Y, W, off, dX)
    want, err = u.mm(Y[R - n:], W[E - 1].t())
    u.assert_within(dX[R - n:], want, u.rounded(want, err, BF16), "last group's gradient")
    assert bool((dX[: R - n] == 0).all())
    del W
    dW = torch.full((E, K, N), 7.0, dtype=BF16, device="cuda")
    ff.ffuse_grouped_gemm_dw(ff.DT_BF16, X, Y, off, dW)
    want, err = u.mm(X[R - n:].t(), Y[R - n:])
    u.assert_within(dW[E - 1], want, u.rounded(want, err, BF16), "last expert's gradient")
    assert bool((dW[: E - 1] == 0).all())


def _layer(gen, sizes, K, N1, N2):
    R, E = sum(sizes), len(sizes)
    return (u.normal(gen, (R, K), 1.0, BF16), u.normal(gen, (E, K, N1), K ** -0.5, BF16), u.normal(gen, (E, K, N1), K ** -0.5, BF16),
            u.normal(gen, (E, N1, N2), N1 ** -0.5, BF16))


def test_a_training_step_in_a_graph_with_new_boundaries_each_replay():
    """Forward, chain and both gradients recorded once; replays read the boundaries and operands they then find."""
    gen, K, N1, N2, R, E = torch.Generator().manual_seed(12), 136, 264, 72, 300, 5
    X, W1, W3, W2 = _layer(gen, [60] * E, K, N1, N2)
    dY, off = u.normal(gen, (R, N1), 1.0, BF16), u.offsets_of([60] * E)
    Y, Z, dX, dW = (torch.empty(s, dtype=BF16, device="cuda") for s in ((R, N1), (R, N2), (R, K), (E, K, N1)))
    ws = torch.empty(ff.ffuse_grouped_workspace_bytes(ff.DT_BF16, R, N1), dtype=torch.uint8, device="cuda")

    def step():
        ff.ffuse_grouped_gemm(ff.DT_BF16, X, W1, W3, off, ff.ACT_SILU, Y)
        ff.ffuse_grouped_ffn(ff.DT_BF16, X, W1, W3, W2, off, ff.ACT_SILU, Z, ws)
        ff.ffuse_grouped_gemm_dx(ff.DT_BF16, dY, W1, off, dX)
        ff.ffuse_grouped_gemm_dw(ff.DT_BF16, X, dY, off, dW)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
    torch.cuda.synchronize()
    for sizes in ([60] * E, [0, 300, 0, 0, 0], [1, 2, 3, 4, 290], [128, 0, 129, 43, 0]):
        off.copy_(u.offsets_of(sizes))
        X.copy_(u.normal(gen, (R, K), 1.0, BF16))
        for t in (Y, Z, dX, dW):
            t.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (Y, Z, dX, dW)]
        torch.randn(1 << 20, device="cuda").sum()
        step()
        torch.cuda.synchronize()
        for a, b in zip(replayed, (Y, Z, dX, dW)):
            assert bool(torch.isfinite(a).all()) and torch.equal(a, b), sizes


def test_two_streams_at_once():
    gen = torch.Generator().manual_seed(13)
    sizes = [[100, 0, 400, 37], [5, 260, 128, 90]]
    layers = [_layer(gen, s, 264, 520, 264) for s in sizes]
    streams = [torch.cuda.Stream() for _ in layers]
    off = [u.offsets_of(s) for s in sizes]
    ws = [torch.empty(ff.ffuse_grouped_workspace_bytes(ff.DT_BF16, sum(s), 520), dtype=torch.uint8, device="cuda") for s in sizes]
    out = [[torch.full((sum(s), 264), float("nan"), dtype=BF16, device="cuda") for _ in range(20)] for s in sizes]
    alone = [torch.empty((sum(s), 264), dtype=BF16, device="cuda") for s in sizes]
    for (X, W1, W3, W2), o, w, y in zip(layers, off, ws, alone):
        ff.ffuse_grouped_ffn(ff.DT_BF16, X, W1, W3, W2, o, ff.ACT_SILU, y, w)
    torch.cuda.synchronize()
    for i in range(20):
        for st, (X, W1, W3, W2), o, w, ys in zip(streams, layers, off, ws, out):
            with torch.cuda.stream(st):
                ff.ffuse_grouped_ffn(ff.DT_BF16, X, W1, W3, W2, o, ff.ACT_SILU, ys[i], w)
    torch.cuda.synchronize()
    for ys, y in zip(out, alone):
        assert all(torch.equal(y, z) for z in ys)


@pytest.mark.parametrize("in_graph", (False, True))
@pytest.mark.parametrize("registered,part", ((False, 1), (False, 2), (True, 1)))
def test_a_workspace_shared_with_the_other_chains(in_graph, registered, part):
    """The chains of one expert remember what they left in a workspace; a grouped chain in between, or replayed
    behind the library's back, makes them clear it again, also where they use only a part of its memory."""
    gen, sizes = torch.Generator().manual_seed(14), [50, 78]
    X, W1, W3, W2 = _layer(gen, sizes, 136, 264, 72)
    plans = [ff.make_plan(ff.FAMILY_REDUCE, bm=128, bh=64, bn2=128, raster=1, splits=(264 + 63) // 64),       # sums that start at zero
             ff.make_plan(ff.FAMILY_TWOPHASE, bm=128, splits=1, raster=2)]                                   # flags that start at zero
    nbytes = 1 << 20
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    off, Y = u.offsets_of(sizes), torch.empty((128, 72), dtype=BF16, device="cuda")
    grouped = lambda: ff.ffuse_grouped_ffn(ff.DT_BF16, X, W1, W3, W2, off, ff.ACT_SILU, Y, ws)  # noqa: E731
    graph = None
    if in_graph:
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            grouped()
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                grouped()
        torch.cuda.synchronize()
    if registered and not in_graph:
        gu.Workspace.buf = None      # (the other tests' registered one)
        ff.ffuse_set_workspace(ws)
    A, B1, B2 = u.normal(gen, (100, 136), 1.0, BF16), u.normal(gen, (136, 264), 136 ** -0.5, BF16), u.normal(gen, (264, 72), 264 ** -0.5, BF16)
    h, eh = u.product64(A, B1, None, ff.ACT_RELU, BF16)
    want, err = u.mm(h, B2)
    err = u.rounded(want, err + eh @ B2.double().abs(), BF16)
    try:
        for plan in plans:
            ff.ffuse_force_plan(plan)
            for _ in range(3):
                Z = torch.full((100, 72), float("nan"), dtype=BF16, device="cuda")
                if registered and not in_graph:
                    ff.ffuse_ffn(A, B1, None, B2, ff.ACT_RELU, Z)
                else:
                    ff.ffuse_ffn_ws(ff.DT_BF16, A, B1, None, B2, ff.ACT_RELU, Z, ws[: nbytes // part])
                assert ff.ffuse_sync_status(check=False) == 0
                u.assert_within(Z, want, err, f"chain of one expert, plan {plan.as_dict()}")
                graph.replay() if graph else grouped()
                torch.cuda.synchronize()
    finally:
        ff.ffuse_force_plan(None)
        if registered and not in_graph:
            ff.ffuse_set_workspace(None)


@pytest.mark.parametrize("sizes,K,N,gated", [
    ([9000, 300, 0, 10700], 136, 4104, False),      # 256 x 256 tiles, several rounds and a rest that is done in parts
    ([9000, 300, 0, 10700], 72, 2056, True),
    ([100] * 23 + [57], 1000, 2056, False),         # 128 x 256, a little over a round
    ([130, 40, 200, 0, 255, 129, 128, 90] * 8, 520, 1416, True),
    ([60, 10, 64, 65, 3] * 20, 264, 2056, False),
    ([129] * 15, 1144, 1144, False),                # 128 x 128, one round and a few tiles in halves
])
def test_forward_and_gradients_of_many_tiles(sizes, K, N, gated):
    """Products of more tiles than the device has CUs, checked in every element: the rests of the rounds, too."""
    gen, R, E, t = torch.Generator().manual_seed(15), sum(sizes) + 2, len(sizes), BF16
    X, W, dY = u.normal(gen, (R, K), 1.0, t), u.normal(gen, (E, K, N), K ** -0.5, t), u.normal(gen, (R, N), 0.1, t)
    W3 = u.normal(gen, (E, K, N), K ** -0.5, t) if gated else None
    off = u.offsets_of(sizes)
    Y, dX, dW = (torch.full(s, 7.0, dtype=t, device="cuda") for s in ((R, N), (R, K), (E, K, N)))
    print("many tiles", len(sizes), R, K, N, gated, flush=True)
    ff.ffuse_grouped_gemm(ff.DT_BF16, X, W, W3, off, ff.ACT_SILU if gated else ff.ACT_IDENTITY, Y)
    ff.ffuse_grouped_gemm_dx(ff.DT_BF16, dY, W, off, dX)
    ff.ffuse_grouped_gemm_dw(ff.DT_BF16, X, dY, off, dW)
    torch.cuda.synchronize()
    for e, s in _spans(sizes):
        want, err = u.product64(X[s], W[e], None if W3 is None else W3[e], ff.ACT_SILU if gated else ff.ACT_IDENTITY, t)
        u.assert_within(Y[s], want, err, f"Y, group {e}")
        want, err = u.mm(dY[s], W[e].t())
        u.assert_within(dX[s], want, u.rounded(want, err, t), f"dX, group {e}")
        want, err = u.mm(X[s].t(), dY[s])
        u.assert_within(dW[e], want, u.rounded(want, err, t), f"dW, group {e}")
    assert bool((Y[R - 2:] == 7).all()) and bool((dX[R - 2:] == 7).all())


def test_weight_gradient_of_large_blocks():
    gen, sizes, K, N = torch.Generator().manual_seed(16), [700, 0, 1301, 64], 1032, 2056
    R = sum(sizes)
    X, dY = u.normal(gen, (R, K), 1.0, F16), u.normal(gen, (R, N), 0.1, F16)
    dW = torch.full((len(sizes), K, N), float("nan"), dtype=F16, device="cuda")
    ff.ffuse_grouped_gemm_dw(ff.DT_F16, X, dY, u.offsets_of(sizes), dW)
    for e, s in _spans(sizes):
        want, err = u.mm(X[s].t(), dY[s])
        u.assert_within(dW[e], want, u.rounded(want, err, F16), f"group {e}")


def test_as_many_groups_as_a_call_takes():
    """1024 groups of about a hundred rows: the largest boundary tables beside the deepest rings."""
    gen, E, K, N = torch.Generator().manual_seed(17), 1024, 72, 2056
    sizes = [(37 * i) % 200 for i in range(E)]
    R = sum(sizes)
    X, dY, W = torch.randn(R, K, device="cuda").to(BF16), torch.randn(R, N, device="cuda").to(BF16), (torch.randn(E, K, N, device="cuda") * K ** -0.5).to(BF16)
    off, Y, dX, dW = u.offsets_of(sizes), torch.empty((R, N), dtype=BF16, device="cuda"), torch.empty((R, K), dtype=BF16, device="cuda"), torch.empty_like(W)
    ff.ffuse_grouped_gemm(ff.DT_BF16, X, W, None, off, ff.ACT_IDENTITY, Y)
    ff.ffuse_grouped_gemm_dx(ff.DT_BF16, dY, W, off, dX)
    ff.ffuse_grouped_gemm_dw(ff.DT_BF16, X, dY, off, dW)
    torch.cuda.synchronize()
    for e, s in _spans(sizes):
        if e % 41 and e not in (1, 63, 64, 1022, 1023):
            continue
        for got, (want, err) in ((Y[s], u.mm(X[s], W[e])), (dX[s], u.mm(dY[s], W[e].t())), (dW[e], u.mm(X[s].t(), dY[s]))):
            u.assert_within(got, want, u.rounded(want, err, BF16), f"group {e}")
    assert bool(torch.isfinite(Y).all()) and bool(torch.isfinite(dX).all()) and bool(torch.isfinite(dW).all())
