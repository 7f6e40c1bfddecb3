"""Workspaces that the chain by expert shares with the chains of one expert: what a call or a replay leaves in one is never
taken for what the next call needs there."""
import pytest
import torch

from paper_2512_12949_amd import binding as ff

import gpu_util as gu
import grouped_util as u

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
K, N1, N2 = 136, 264, 72
SUMS = ff.make_plan(ff.FAMILY_REDUCE, bm=128, bh=64, bn2=128, raster=1, splits=(N1 + 63) // 64)      # sums that start at zero
FLAGS = ff.make_plan(ff.FAMILY_TWOPHASE, bm=128, splits=1, raster=2)                               # flags that start at zero


class _Work:
    """A chain by expert, and one of one expert with the error it may have."""

    def __init__(self, seed):
        gen, sizes = torch.Generator().manual_seed(seed), [50, 78]
        self.R = R = sum(sizes)
        self.X, self.W1, self.W3 = u.normal(gen, (R, K), 1.0, BF16), u.normal(gen, (2, K, N1), K ** -0.5, BF16), u.normal(gen, (2, K, N1), K ** -0.5, BF16)
        self.W2, self.off, self.Y = u.normal(gen, (2, N1, N2), N1 ** -0.5, BF16), u.offsets_of(sizes), torch.empty((R, N2), dtype=BF16, device="cuda")
        self.A, self.B1, self.B2 = u.normal(gen, (100, K), 1.0, BF16), u.normal(gen, (K, N1), K ** -0.5, BF16), u.normal(gen, (N1, N2), N1 ** -0.5, BF16)
        h, eh = u.product64(self.A, self.B1, None, ff.ACT_RELU, BF16)
        self.want, err = u.mm(h, self.B2)
        self.err = u.rounded(self.want, err + eh @ self.B2.double().abs(), BF16)

    def grouped(self, ws):
        ff.ffuse_grouped_ffn(ff.DT_BF16, self.X, self.W1, self.W3, self.W2, self.off, ff.ACT_SILU, self.Y, ws)

    def recorded(self, call):
        """A graph of one call."""
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                call()
        torch.cuda.synchronize()
        return graph

    def chain(self, plan, ws, what):
        """The chain of one expert in workspace `ws` (None: the registered one), checked."""
        Z = torch.full((100, N2), float("nan"), dtype=BF16, device="cuda")
        ff.ffuse_force_plan(plan)
        try:
            if ws is None:
                ff.ffuse_ffn(self.A, self.B1, None, self.B2, ff.ACT_RELU, Z)
            else:
                ff.ffuse_ffn_ws(ff.DT_BF16, self.A, self.B1, None, self.B2, ff.ACT_RELU, Z, ws)
            assert ff.ffuse_sync_status(check=False) == 0, what
        finally:
            ff.ffuse_force_plan(None)
        u.assert_within(Z, self.want, self.err, what)


def _workspace():
    return torch.empty(1 << 20, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("count", (1, 9, 20))
def test_more_recorded_workspaces_than_are_remembered(count):
    w = _Work(30)
    w.grouped(_workspace())
    spaces = [_workspace() for _ in range(count)]
    graphs = [w.recorded(lambda ws=ws: w.grouped(ws)) for ws in spaces]
    for i in sorted({0, count // 2, count - 1}):
        for plan in (SUMS, FLAGS):
            for step in range(3):
                w.chain(plan, spaces[i], f"workspace {i} of {count}, step {step}")
                graphs[i].replay()
                torch.cuda.synchronize()


def test_a_registered_workspace_that_a_graph_uses():
    """By the registered workspace's calls, by others that name it, and after it is registered no more."""
    w, ws = _Work(31), _workspace()
    gu.Workspace.buf = None      # (the other tests' registered one)
    ff.ffuse_set_workspace(ws)
    try:
        w.grouped(ws)
        graph = w.recorded(lambda: w.grouped(ws))
        for space in (None, ws, ws[: 1 << 19]):
            for plan in (SUMS, FLAGS):
                for step in range(3):
                    w.chain(plan, space, f"{'registered' if space is None else space.numel()}, step {step}")
                    graph.replay()
                    torch.cuda.synchronize()
    finally:
        ff.ffuse_set_workspace(None)
    for plan in (SUMS, FLAGS):
        for step in range(3):
            w.chain(plan, ws, f"no longer registered, step {step}")
            graph.replay()
            torch.cuda.synchronize()


@pytest.mark.parametrize("whole", ("eager", "recorded", "registered", "grouped"))
def test_the_whole_of_a_workspace_after_its_half(whole):
    """What is remembered of the half does not outlive a call on the whole."""
    w, ws = _Work(32), _workspace()
    half = ws[: 1 << 19]
    for first, other in ((SUMS, FLAGS), (FLAGS, SUMS)):
        w.chain(first, half, "half")
        w.chain(first, half, "half, again")
        use = {"grouped": lambda: w.grouped(ws), "recorded": lambda: w.chain(other, ws, "whole")}.get(whole, lambda: w.chain(other, ws, "whole"))
        if whole == "recorded":
            Z = torch.empty((100, N2), dtype=BF16, device="cuda")
            ff.ffuse_force_plan(other)
            try:
                use = w.recorded(lambda: ff.ffuse_ffn_ws(ff.DT_BF16, w.A, w.B1, None, w.B2, ff.ACT_RELU, Z, ws)).replay
            finally:
                ff.ffuse_force_plan(None)
        elif whole == "registered":
            gu.Workspace.buf = None
            ff.ffuse_set_workspace(ws)
            w.chain(first, half, "half of the registered one")
            use = lambda: w.chain(other, None, "registered")  # noqa: E731
        for step in range(3):
            use()
            torch.cuda.synchronize()
            w.chain(first, half, f"half after the whole, {whole}, step {step}")
        if whole == "registered":
            ff.ffuse_set_workspace(None)


def test_the_fp32_path_of_two_launches_in_a_graph():
    """Its intermediate, written by replays, over another chain's sums."""
    w, ws = _Work(33), _workspace()
    A, B1, B2 = (torch.ones(s, device="cuda") for s in ((100, K), (K, N1), (N1, N2)))
    Z = torch.empty((100, N2), device="cuda")
    graph = w.recorded(lambda: ff.ffuse_ffn_unfused_ws(ff.DT_F32, A, B1, None, B2, ff.ACT_RELU, Z, ws))
    for plan in (SUMS, FLAGS):
        for step in range(3):
            w.chain(plan, ws, f"step {step}")
            graph.replay()
            torch.cuda.synchronize()
            assert bool((Z == K * N1).all())


def test_a_status_is_no_part_of_an_intermediate():
    """ffuse_sync_status after a chain by expert, and after a replay of one, in the workspace of a two-phase call."""
    w, ws = _Work(34), _workspace()
    graph = w.recorded(lambda: w.grouped(ws))
    w.chain(FLAGS, ws, "before")
    w.grouped(ws)
    assert ff.ffuse_sync_status(check=False) == 0
    w.chain(FLAGS, ws, "between")
    graph.replay()
    torch.cuda.synchronize()
    assert ff.ffuse_sync_status(check=False) == 0
