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
    return lib.ffuse_grouped_ffn(0, X.at, W.at, None, W.at, OFF.at, ff.ACT_SILU, M, 2, K, N1, N2, Y.at, ws.at, ws.bytes, None)


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
