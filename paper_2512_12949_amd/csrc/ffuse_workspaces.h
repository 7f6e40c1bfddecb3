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
    void forget() { zero = 0; small_flags = nullptr; }
    bool overlaps(const void* p, size_t n) const {
        const char *a = static_cast<const char*>(p), *b = static_cast<const char*>(ptr);
        return ptr && a < b + bytes && b < a + n;
    }
};

// A set of addresses, as ranges in rising order that do not touch.  It never loses one: when it is full, the two ranges with the
// least between them become one, and what lies between counts as in the set.
class AddressRanges {
public:
    bool meets(const void* p, size_t bytes) const {
        const uintptr_t from = reinterpret_cast<uintptr_t>(p), to = from + bytes;
        for (int i = 0; i < n_; ++i)
            if (r_[i].from < to && from < r_[i].to) return true;
        return false;
    }
    void add(const void* p, size_t bytes) {
        Range x{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes};
        if (bytes == 0) return;
        int i = 0, end;
        while (i < n_ && r_[i].to < x.from) ++i;
        for (end = i; end < n_ && r_[end].from <= x.to; ++end) {
            if (r_[end].from < x.from) x.from = r_[end].from;
            if (r_[end].to > x.to) x.to = r_[end].to;
        }
        replace(i, end, &x, 1);
    }
    void remove(const void* p, size_t bytes) {
        const uintptr_t from = reinterpret_cast<uintptr_t>(p), to = from + bytes;
        for (int i = 0; i < n_;) {
            const Range x = r_[i];
            Range left[2];
            int n = 0;
            if (x.from < from) left[n++] = Range{x.from, x.to < from ? x.to : from};
            if (x.to > to) left[n++] = Range{x.from > to ? x.from : to, x.to};
            if (n == 2 && n_ == kMost) return;   // (no room for both ends: all of it stays)
            replace(i, i + 1, left, n);
            i += n;
        }
    }

private:
    struct Range { uintptr_t from, to; };
    static constexpr int kMost = 256;
    Range r_[kMost + 1];
    int n_ = 0;

    // ranges i .. end - 1 by `count` others
    void replace(int i, int end, const Range* with, int count) {
        const int move = count - (end - i);
        if (move < 0) for (int j = end; j < n_; ++j) r_[j + move] = r_[j];
        else for (int j = n_ - 1; j >= end; --j) r_[j + move] = r_[j];
        for (int j = 0; j < count; ++j) r_[i + j] = with[j];
        n_ += move;
        if (n_ <= kMost) return;
        int least = 1;
        for (int j = 2; j < n_; ++j)
            if (r_[j].from - r_[j - 1].to < r_[least].from - r_[least - 1].to) least = j;
        r_[least - 1].to = r_[least].to;
        for (int j = least + 1; j < n_; ++j) r_[j - 1] = r_[j];
        --n_;
    }
};

struct Workspaces {
    Workspace reg;           // the workspace registered with ffuse_set_workspace
    Workspace seen[8];       // workspaces passed per call (ffuse_ffn_ws ...), most recently used kept
    uint64_t clock = 0;
    AddressRanges recorded;  // workspaces of calls that were recorded into graphs: replays the library does not see may
                             // dirty them at any time, so nothing is remembered of a workspace that one of them overlaps

    // the record of a per-call workspace
    Workspace& named(void* ptr, size_t bytes) {
        Workspace* oldest = &seen[0];
        for (Workspace& w : seen) {
            if (w.ptr == ptr && w.bytes == bytes) { w.used = ++clock; return w; }
            if (w.used < oldest->used) oldest = &w;
        }
        *oldest = Workspace{ptr, bytes, 0, nullptr, ++clock};
        return *oldest;
    }
    // [ptr, ptr + bytes) becomes the registered workspace: its memory may have been in other hands in between, and graphs that used
    // it are no more.  It is cleared now, or, into_graph, whenever the graph is replayed.
    void registered(void* ptr, size_t bytes, bool into_graph) {
        for (Workspace& w : seen)
            if (w.overlaps(ptr, bytes)) w = Workspace{};
        recorded.remove(ptr, bytes);
        if (into_graph) recorded.add(ptr, bytes);
        reg = Workspace{ptr, bytes, into_graph ? 0 : bytes, nullptr, 0};
    }
    void unregistered() { reg = Workspace{}; }

    // A call that runs in `w`, recorded into a graph or not, from before its first launch to after its last.  What is known of
    // other records that share memory with it no longer holds.  (Whatever a call on a workspace that a graph uses leaves behind, a
    // replay may find something else.)
    void begin(Workspace& w, bool into_graph) {
        overwritten(w.ptr, w.bytes, into_graph, &w);
        end(w);
    }
    void end(Workspace& w) {
        if (recorded.meets(w.ptr, w.bytes)) w.forget();
    }
    // A call, recorded into a graph or not, writes into [ptr, ptr + bytes); `own`: the record, if any, that it keeps itself.
    void overwritten(void* ptr, size_t bytes, bool into_graph, const Workspace* own = nullptr) {
        if (into_graph) recorded.add(ptr, bytes);
        if (&reg != own && reg.overlaps(ptr, bytes)) reg.forget();
        for (Workspace& w : seen)
            if (&w != own && w.overlaps(ptr, bytes)) w.forget();
    }
};

}  // namespace ffuse
