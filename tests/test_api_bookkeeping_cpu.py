"""What the C interface does between its launches, over launches that are lines in a log."""
import ctypes
import threading
import time

import pytest

from paper_2512_12949_amd import binding as ff

import api_stub

M, K, N1, N2 = 100, 136, 264, 72
SUMS = ff.make_plan(ff.FAMILY_REDUCE, bm=128, bh=64, bn2=128, raster=1, splits=(N1 + 63) // 64)


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return api_stub.build(tmp_path_factory.mktemp("stub"))


class _Space:
    """16-byte aligned memory of a size that everything here fits in."""

    def __init__(self, nbytes=1 << 20):
        self.raw = ctypes.create_string_buffer(nbytes + 16)
        self.at = (ctypes.addressof(self.raw) + 15) & ~15
        self.bytes = nbytes


X, W, Y, OFF = _Space(), _Space(), _Space(), _Space()


def _grouped(lib, ws):
    return lib.ffuse_grouped_ffn(0, X.at, W.at, None, W.at, OFF.at, ff.ACT_SILU, 2 * M, 2, K, N1, N2, Y.at, ws.at, ws.bytes, None)


def _chain(lib, ws, plan):
    assert lib.ffuse_force_plan(ctypes.byref(plan)) == 0
    return lib.ffuse_ffn_ws(0, X.at, W.at, None, W.at, ff.ACT_RELU, M, K, N1, N2, Y.at, ws.at, ws.bytes, None)


def test_no_call_gets_between_the_bookkeeping_of_a_chain_by_expert_and_its_launches(lib):
    """Two host threads with one workspace and one stream: whoever comes second finds the workspace as the first's launches leave it."""
    ws = _Space()
    lib.stub_reset(b"", 0)
    assert _chain(lib, ws, SUMS) == 0 and _chain(lib, ws, SUMS) == 0
    assert api_stub.log(lib) == ["zero", "reduce", "finalize", "reduce", "finalize"]
    lib.stub_reset(b"grouped", 0)
    first = threading.Thread(target=_grouped, args=(lib, ws))
    first.start()
    end = time.time() + 20
    while not lib.stub_held() and time.time() < end:
        time.sleep(0.001)
    assert _chain(lib, ws, SUMS) == 0
    first.join()
    assert api_stub.log(lib) == ["grouped", "held", "grouped", "zero", "reduce", "finalize"]


FLAGS = ff.make_plan(ff.FAMILY_TWOPHASE, bm=128, splits=1, raster=2)


@pytest.mark.parametrize("replayed", (False, True))
def test_no_status_is_read_from_what_a_chain_by_expert_wrote(lib, replayed):
    """The verdict of a two-phase launch lies in its workspace; an intermediate written over it, by a call or by a replay behind the
    library's back, says nothing about that launch."""
    ws = _Space()
    lib.stub_reset(b"", 0)
    assert _chain(lib, ws, FLAGS) == 0 and lib.ffuse_sync_status(None) == 0
    if replayed:
        ctypes.memset(ws.at, 0x3f, 2 * M * N1 * 2)
    else:
        assert _grouped(lib, ws) == 0
    assert lib.ffuse_sync_status(None) == 0
    assert _chain(lib, ws, FLAGS) == 0 and _chain(lib, ws, FLAGS) == 0 and lib.ffuse_sync_status(None) == 0


@pytest.mark.parametrize("word,status", ((0, 0), (1, -9), (2, -10), (3, -10)))
def test_a_verdict_is_reported(lib, word, status):
    ws = _Space()
    lib.stub_reset(b"", 0)
    assert _chain(lib, ws, FLAGS) == 0
    flags = ws.at + (2 * M * N1 + 255) // 256 * 256
    ctypes.c_uint32.from_address(flags + 12).value = word
    assert lib.ffuse_sync_status(None) == status
    other = _Space()      # (a chain by expert elsewhere does not hide it)
    assert _grouped(lib, other) == 0 and lib.ffuse_sync_status(None) == status
