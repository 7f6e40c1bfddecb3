// What the library remembers about caller-owned workspaces between calls.  Host code without any device call: the
// caller holds the library's lock.
#pragma once
#include <cstddef>
#include <cstdint>

namespace ffuse {

// How much of a workspace's start is known to be zero (the reduce family keeps its sums there) and where the two-phase
// family last left clean barrier flags.  A workspace the library has not seen (or whose size changed) counts as dirty.
struct Workspace {
    void* ptr = nullptr;
    size_t bytes = 0;
    size_t zero = 0;                  // bytes at the start known to be zero
    uint32_t* small_flags = nullptr;  // where the two-phase family last left clean barrier flags
    uint64_t used = 0;                // age, for replacement
    bool in_graph = false;            // a call on this workspace was recorded into a graph: replays the library does
                                      // not see may dirty it at any time, so nothing above is trusted any more
    void forget() { zero = 0; small_flags = nullptr; }
    bool overlaps(const void* p, size_t n) const {
        const char *a = static_cast<const char*>(p), *b = static_cast<const char*>(ptr);
        return ptr && a < b + bytes && b < a + n;
    }
};

struct Workspaces {
    Workspace reg;           // the workspace registered with ffuse_set_workspace
    Workspace seen[8];       // workspaces passed per call (ffuse_ffn_ws ...), most recently used kept
    uint64_t clock = 0;

    // The record of a per-call workspace.  Part of a workspace that a graph uses is one itself, and the records of those are
    // replaced last.
    Workspace& named(void* ptr, size_t bytes) {
        Workspace* oldest = &seen[0];
        bool in_graph = reg.in_graph && reg.overlaps(ptr, bytes);
        for (Workspace& w : seen) {
            if (w.ptr == ptr && w.bytes == bytes) { w.used = ++clock; return w; }
            in_graph = in_graph || (w.in_graph && w.overlaps(ptr, bytes));
            if (w.in_graph != oldest->in_graph ? oldest->in_graph : w.used < oldest->used) oldest = &w;
        }
        *oldest = Workspace{ptr, bytes, 0, nullptr, ++clock, in_graph};
        return *oldest;
    }
    // [ptr, ptr + bytes), all zeros, becomes the registered workspace: its memory may have been in other hands in between
    void registered(void* ptr, size_t bytes) {
        for (Workspace& w : seen)
            if (w.overlaps(ptr, bytes)) w = Workspace{};
        reg = Workspace{ptr, bytes, bytes, nullptr, 0, false};
    }
    void unregistered() { reg = Workspace{}; }

    // A call that runs in `w`, recorded into a graph or not, from before its first launch to after its last.  (Whatever a call on
    // a workspace that a graph uses leaves behind, a replay may find something else.)
    void begin(Workspace& w, bool recorded) {
        if (recorded) w.in_graph = true;
        end(w);
    }
    void end(Workspace& w) {
        if (w.in_graph) w.forget();
    }
    // a call of another kind, recorded into a graph or not, writes into [ptr, ptr + bytes)
    void overwritten(void* ptr, size_t bytes, bool recorded) {
        if (recorded) named(ptr, bytes);   // (so that a later call on it knows)
        const auto dirty = [&](Workspace& w) {
            if (!w.overlaps(ptr, bytes)) return;
            w.forget();
            if (recorded) w.in_graph = true;
        };
        dirty(reg);
        for (Workspace& w : seen) dirty(w);
    }
};

}  // namespace ffuse
