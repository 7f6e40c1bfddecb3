"""What the library remembers about workspaces between calls, against a model of the memory itself: a call may skip a
clearing only where the memory really is as it needs it."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_12949_amd", "csrc")
DRIVER = """
#include "ffuse_workspaces.h"
namespace { ffuse::Workspaces ws; }
extern "C" {
void reset() { ws = ffuse::Workspaces(); }
// the records' side of a call: bytes == 0 for the registered workspace
static ffuse::Workspace& of(char* p, size_t bytes) { return bytes ? ws.named(p, bytes) : ws.reg; }
// sums in the first `need` bytes, which start at zero and are zero again afterwards: 1 where they are cleared first
int sums(char* p, size_t bytes, size_t need, int recorded) {
    ffuse::Workspace& w = of(p, bytes);
    ws.begin(w, recorded);
    const int clears = w.zero < need;
    if (clears) w.zero = need;
    w.small_flags = nullptr;
    ws.end(w);
    return clears;
}
// `at` bytes of data and flags behind them, which start clean and are left clean: 1 where they are cleared first
int flags(char* p, size_t bytes, size_t at, int recorded) {
    ffuse::Workspace& w = of(p, bytes);
    ws.begin(w, recorded);
    uint32_t* f = reinterpret_cast<uint32_t*>(static_cast<char*>(w.ptr) + at);
    const int clears = w.small_flags != f;
    w.small_flags = f;
    w.zero = 0;
    ws.end(w);
    return clears;
}
void overwritten(char* p, size_t bytes, int recorded) { ws.overwritten(p, bytes, recorded); }
void registered(char* p, size_t bytes, int recorded) { ws.registered(p, bytes, recorded); }
void unregistered() { ws.unregistered(); }
static ffuse::AddressRanges ranges;
void ranges_reset() { ranges = ffuse::AddressRanges(); }
void ranges_add(char* p, size_t bytes) { ranges.add(p, bytes); }
void ranges_remove(char* p, size_t bytes) { ranges.remove(p, bytes); }
int ranges_meet(char* p, size_t bytes) { return ranges.meets(p, bytes); }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("records")
    (d / "driver.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(d / "driver.cpp"), "-o", str(d / "driver.so")], check=True)
    L = ctypes.CDLL(str(d / "driver.so"))
    n, p, i = ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int
    for name, args in (("reset", []), ("sums", [p, n, n, i]), ("flags", [p, n, n, i]), ("overwritten", [p, n, i]), ("registered", [p, n, i]), ("unregistered", []),
                       ("ranges_reset", []), ("ranges_add", [p, n]), ("ranges_remove", [p, n]), ("ranges_meet", [p, n])):
        getattr(L, name).argtypes = args
    L.reset()
    return L


BASE, SIZE = 1 << 20, 1 << 12      # never dereferenced


def _place(i):
    return BASE + i * SIZE


@pytest.mark.parametrize("count", (1, 8, 9, 40, 1000))
@pytest.mark.parametrize("kind", ("overwritten", "sums", "flags"))
def test_a_recorded_workspace_stays_one(lib, count, kind):
    """However many workspaces graphs use: after a replay, which nobody sees, each of them is cleared again."""
    lib.reset()
    for i in range(count):
        getattr(lib, kind)(_place(i), SIZE, *(() if kind == "overwritten" else (256,)), 1)
    for i in (0, count // 2, count - 1):
        for call in (lib.sums, lib.flags):
            assert [call(_place(i), SIZE, 512, 0) for _ in range(3)] == [1, 1, 1]      # (a replay in between each)


def test_recorded_workspaces_take_no_place_from_others(lib):
    """Workspaces in use by turns are cleared once, whatever graphs use beside them."""
    for recorded in (0, 7, 8, 30):
        lib.reset()
        for i in range(recorded):
            lib.overwritten(_place(100 + 2 * i), SIZE, 1)
        assert sum(lib.sums(_place(i % 2), SIZE, 512, 0) for i in range(20)) == 2, recorded


@pytest.mark.parametrize("seed", range(6))
def test_a_set_of_address_ranges(lib, seed):
    """Against a plain set of addresses, in no more ranges than there is room for: exactly the same."""
    rng, has = random.Random(seed), set()
    lib.ranges_reset()
    for _ in range(400):
        at = rng.randrange(1, 600)
        n = rng.choice((0, 1, 2, 5, 40))
        if rng.random() < 0.6:
            lib.ranges_add(at, n)
            has |= set(range(at, at + n))
        else:
            lib.ranges_remove(at, n)
            has -= set(range(at, at + n))
        assert [bool(lib.ranges_meet(a, 1)) for a in range(1, 650)] == [a in has for a in range(1, 650)]
        a, n = rng.randrange(1, 600), rng.randrange(1, 50)
        assert bool(lib.ranges_meet(a, n)) == any(x in has for x in range(a, a + n))


def test_a_full_set_of_address_ranges_loses_none(lib):
    rng, has = random.Random(7), set()
    lib.ranges_reset()
    for _ in range(3000):
        a = 10 * rng.randrange(1, 4000)
        lib.ranges_add(a, 5)
        has |= set(range(a, a + 5))
    lib.ranges_remove(10002, 1)
    has.discard(10002)
    assert all(lib.ranges_meet(a, 1) for a in has)
    assert not lib.ranges_meet(5, 4) and not lib.ranges_meet(45000, 1000)
    lib.ranges_remove(1, 50000)
    assert not lib.ranges_meet(1, 50000)


def test_registering_is_the_end_of_graphs(lib):
    """ffuse_set_workspace hands memory over: it is cleared there, and remembered again, as far as the registered workspace goes."""
    lib.reset()
    lib.overwritten(_place(0), 4 * SIZE, 1)
    lib.registered(_place(1), SIZE, 0)
    assert [lib.sums(None, 0, 512, 0) for _ in range(3)] == [0, 0, 0]
    assert [lib.sums(_place(2), SIZE, 512, 0) for _ in range(3)] == [1, 1, 1]
    lib.unregistered()
    assert [lib.sums(_place(1), SIZE, 512, 0) for _ in range(3)] == [1, 0, 0]
    assert [lib.sums(_place(0), SIZE, 512, 0) for _ in range(3)] == [1, 1, 1]


def test_a_recorded_registered_workspace_stays_one(lib):
    """Whoever names its memory afterwards, and after it is registered no more."""
    lib.reset()
    lib.registered(_place(0), SIZE, 0)
    lib.sums(None, 0, 512, 1)
    assert [lib.sums(None, 0, 512, 0) for _ in range(3)] == [1, 1, 1]
    assert [lib.sums(_place(0), SIZE // 2, 512, 0) for _ in range(3)] == [1, 1, 1]
    lib.unregistered()
    assert [lib.sums(_place(0), SIZE, 512, 0) for _ in range(3)] == [1, 1, 1]


class _Memory:
    """What really lies in memory, a letter a word of 64 bytes, beside what the records say.  A call that leaves out its clearing where
    it should not have fails here."""
    WORDS, WORD = 64, 64

    def __init__(self, lib):
        lib.reset()
        self.lib, self.words, self.reg, self.graphs = lib, ["?"] * self.WORDS, None, []

    def call(self, kind, space, need, into_graph=False):
        """space: (first word, words), or None for the registered one; need: words of sums, or of data before the flags."""
        first, n = space or self.reg
        args = (BASE + first * self.WORD, n * self.WORD) if space else (None, 0)
        if kind == "grouped":
            self.lib.overwritten(BASE + first * self.WORD, n * self.WORD, into_graph)
            todo = [("H", first, need)]
        else:
            clears = getattr(self.lib, kind)(*args, need * self.WORD, into_graph)
            if kind == "sums":
                todo = ([("0", first, need)] if clears else []) + [("0?", first, need)]
            else:      # (clean flags are zeros; what is zero may as well be flags)
                todo = ([("0", first + need, 1)] if clears else []) + [("0?", first + need, 1), ("H", first, need)]
        if into_graph:
            assert kind == "grouped" or clears
            self.graphs.append(todo)
        else:
            self.run(todo)

    def run(self, todo):
        for what, first, n in todo:
            if what == "0?":
                assert self.words[first:first + n] == ["0"] * n, f"{n} words from {first} on are not zero: {self.words}"
            else:
                self.words[first:first + n] = [what] * n

    def register(self, first, n):
        self.lib.registered(BASE + first * self.WORD, n * self.WORD, 0)
        self.words[first:first + n] = ["0"] * n
        self.reg, self.graphs = (first, n), [g for g in self.graphs if all(a + k <= first or first + n <= a for _, a, k in g)]


@pytest.mark.parametrize("kind", ("grouped", "sums", "flags"))
@pytest.mark.parametrize("into_graph", (False, True))
def test_a_call_on_the_whole_of_a_workspace_is_one_on_its_half(lib, kind, into_graph):
    """The half's record, and the registered workspace's, are there before the whole is used."""
    m = _Memory(lib)
    m.register(40, 8)
    for _ in range(2):
        m.call("sums", (0, 8), 4)
        m.call("sums", None, 4)
    m.call(kind, (0, 16), 12, into_graph)
    m.call(kind, (32, 24), 20, into_graph)
    for g in m.graphs:
        m.run(g)
    m.call("sums", (0, 8), 4)
    m.call("sums", None, 4)
    for g in m.graphs:
        m.run(g)
    m.call("sums", (0, 8), 4)
    m.call("sums", None, 4)


def test_another_size_hands_a_workspace_over(lib):
    """Also a size that was named before."""
    m = _Memory(lib)
    for _ in range(4):
        for n in (16, 12):
            m.words[0:16] = ["the caller's"] * 16
            m.call("sums", (0, n), 8)


@pytest.mark.parametrize("seed", range(40))
def test_calls_and_replays_in_any_order(lib, seed):
    """Workspaces that overlap or not, used by turns, recorded, replayed and registered: whatever is left out was not needed."""
    rng, m = random.Random(seed), _Memory(lib)
    spaces = [(first, n) for first, n in ((rng.randrange(0, 48), rng.choice((4, 6, 8, 12, 16))) for _ in range(rng.choice((2, 4, 14))))]
    m.register(*rng.choice(spaces))
    for _ in range(400):
        what = rng.random()
        if what < 0.06 and m.graphs:
            m.run(rng.choice(m.graphs))
        elif what < 0.08:
            m.register(*rng.choice(spaces))
        else:
            space = None if rng.random() < 0.2 else rng.choice(spaces)
            m.call(rng.choice(("sums", "sums", "flags", "grouped")), space if space or what < 0.5 else m.reg, rng.randrange(1, (space or m.reg)[1]),
                   into_graph=seed % 2 == 1 and rng.random() < 0.02)


def test_registered_while_recording(lib):
    """Its clearing is part of the graph: nothing has been cleared yet, and a replay clears sums at any time."""
    lib.reset()
    lib.registered(_place(0), SIZE, 1)
    assert [lib.sums(None, 0, 512, 0) for _ in range(3)] == [1, 1, 1]
