// Rows grouped by expert: what the kernels that multiply each group of rows by a matrix of its own share -- the
// group boundaries, read on the device, and the map from work items to (group, row block, column block).
//
// offsets[0 .. E] are the boundaries: group e is rows offsets[e] .. offsets[e + 1] - 1.  They are data, so nothing
// the host has checked: a boundary is clamped to 0 .. R and to the largest one before it, which makes every group a
// range inside the tensor, and the groups disjoint, whatever the values are.
#pragma once
#include "ffuse_dev.h"

namespace ffuse {

static constexpr int kMaxGroups = 1024;   // groups of a call: their boundaries are kept in LDS
static constexpr int kGroupBand = 8;      // row blocks that share their column blocks in an XCD's L2 at a time

// LDS bytes of the tables below
__host__ __device__ constexpr int group_table_bytes(int E) { return 8 * E; }
// LDS that the kernels' own arrays may take beside the largest tables (160 KB in all)
static constexpr int kLdsBesideGroups = 160 * 1024 - group_table_bytes(kMaxGroups);
// groups whose tables leave a CU room for `per_cu` workgroups with `lds` bytes of arrays of their own
constexpr int most_groups(int lds, int per_cu) { return (160 * 1024 / per_cu - lds) / group_table_bytes(1); }

struct Groups {
    int* start;   // [E]: the clamped boundaries
    int* tiles;   // [E]: row blocks of the groups up to and including this one
    int E, end;   // end: the last boundary
};

// Fills the tables; the whole workgroup calls it, the first wave works.  offsets == nullptr: one group of all R rows.
// scratch: 4 bytes of LDS that are free again afterwards.
__device__ __forceinline__ void scan_groups(Groups& g, char* table, char* scratch, const int32_t* offsets, int E, int R, int bm, int tid) {
    g.start = reinterpret_cast<int*>(table);
    g.tiles = g.start + E;
    g.E = E;
    if (tid < 64) {
        int most = 0, sum = 0;   // of the groups before this round of 64
        for (int base = 0; base < E; base += 64) {
            const int e = base + tid;
            const bool live = e < E;
            int lo = 0, hi = R;
            if (offsets) {
                lo = live ? min(max(offsets[e], 0), R) : 0;
                hi = live ? min(max(offsets[e + 1], 0), R) : 0;
            }
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int up = __shfl_up(lo, d);
                if (tid >= d) lo = max(lo, up);
            }
            lo = max(lo, most);
            hi = max(lo, hi);
            int n = live ? (hi - lo + bm - 1) / bm : 0;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int up = __shfl_up(n, d);
                if (tid >= d) n += up;
            }
            n += sum;
            if (live) {
                g.start[e] = lo;
                g.tiles[e] = n;
                if (e == E - 1) *reinterpret_cast<int*>(scratch) = hi;
            }
            most = __shfl(lo, 63);
            sum = __shfl(n, 63);
        }
    }
    __syncthreads();

    g.end = __builtin_amdgcn_readfirstlane(*reinterpret_cast<int*>(scratch));
    __syncthreads();
}

struct GroupItem {
    int e;           // group
    int64_t row0;    // first row of the block
    int rows;        // rows of the group from there on (more than the block holds, or fewer)
    int col;         // first column
};

// Items of `bm` rows x `bn` columns, `ncol` column blocks.  Those of an XCD are consecutive, the row blocks of a group in bands
// of kGroupBand, column block by column block, so that the 32 workgroups of an XCD work on a patch of a band and a few column
// blocks and fetch each panel of either operand into its L2 once.
__device__ __forceinline__ int group_items(const Groups& g, int ncol, int xcd) {   // of an XCD
    const int total = __builtin_amdgcn_readfirstlane(g.tiles[g.E - 1]) * ncol, per = (total + 7) >> 3;
    return min(per, max(total - xcd * per, 0));
}
__device__ __forceinline__ GroupItem group_item(const Groups& g, int bm, int bn, int ncol, int xcd, int idx) {   // idx < group_items
    const int total = __builtin_amdgcn_readfirstlane(g.tiles[g.E - 1]) * ncol;
    const int v = xcd * ((total + 7) >> 3) + idx;
    const int lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    int e = 0;       // groups that end at or before the item
    for (int base = 0; base < g.E; base += 64) {
        const int i = base + lane;
        const uint64_t before = __ballot(i < g.E && g.tiles[i < g.E ? i : 0] * ncol <= v);
        e += __popcll(before);
        if (before != ~0ull) break;
    }
    e = __builtin_amdgcn_readfirstlane(e);
    const int t0 = __builtin_amdgcn_readfirstlane(e ? g.tiles[e - 1] : 0), nt = __builtin_amdgcn_readfirstlane(g.tiles[e]) - t0;
    const int w = v - t0 * ncol, band = w / (kGroupBand * ncol), in = w - band * kGroupBand * ncol;
    const int h = min(kGroupBand, nt - band * kGroupBand);
    const int c = in / h, r = band * kGroupBand + in - c * h;
    const int first = __builtin_amdgcn_readfirstlane(g.start[e]), last = __builtin_amdgcn_readfirstlane(e + 1 < g.E ? g.start[e + 1] : g.end);
    return {e, (int64_t)first + (int64_t)r * bm, last - first - r * bm, c * bn};
}

// One workgroup's share of an XCD's items: `count` of them, numbers loc, loc + step, ...; or, PARTS > 1, of the parts (PM rows x PN
// columns) of the `count` items from `first` on.
template <int PM, int PN, int PARTS> struct ItemWalk {
    const Groups& g;
    int bm, bn, ncol, cols, xcd, first, count, step, at;
    __device__ __forceinline__ bool next(GroupItem& it) {
        for (; at < count * PARTS; at += step) {
            it = group_item(g, bm, bn, ncol, xcd, first + at / PARTS);
            if (PARTS > 1) {
                const int part = at % PARTS, down = bm / PM;
                it.row0 += part % down * PM;
                it.rows -= part % down * PM;
                it.col += part / down * PN;
                if (it.rows <= 0 || it.col >= cols) continue;
            }
            at += step;
            return true;
        }
        return false;
    }
};

// The items of an XCD that its workgroups cannot all have one of: they are done in parts, where that is sooner (a part takes
// `cost` of an item's time).  Returns the items that are left whole.
template <int PARTS> __device__ __forceinline__ int whole_items(int items, int step, float cost) {
    const int left = items % step;
    if (items < step || left == 0) return items;
    return (float)((left * PARTS + step - 1) / step) * cost < 0.95f ? items - left : items;
}

// ---- host side of the launches
// row blocks of bm rows that R rows in at most E groups can come to: a group has a row at least
inline int64_t most_row_blocks(int64_t R, int64_t E, int bm) {
    const int64_t groups = R < E ? R : E;
    return groups + (R - groups) / bm;
}
// persistent workgroups: as many as fit, a multiple of eight (an XCD each), no more than there can be items
inline int persistent_grid(int64_t items, int cus, int per_cu) {
    const int64_t most = (int64_t)cus * per_cu;
    const int64_t n = items < most ? items : most;
    return (int)((n + 7) / 8 * 8);
}

// A tile that a kernel is built for, and what an item of it takes: `step` us for each 128 bytes of the contraction, measured
// with every CU at work on `per_cu` items of a large problem, and `fixed` us beside them.  Left-over items are done in `parts`
// parts of `cost` of an item's time (whole_items; 1: they are not).
struct Tile {
    int bm, bn, per_cu;
    float step, fixed;
    int parts;
    float cost;
};
// The tile whose rounds of items take the least time.  Where the boundaries are known on the device alone, every group
// is taken to have the average number of rows and half a block more, and the last round to be as full as rounds are on average.
template <int N> int pick_tile(const Tile (&tiles)[N], int64_t R, int64_t E, int64_t cols, int64_t bytes, int cus, int without = -1) {
    int best = -1;
    double least = 0.0;
    for (int i = 0; i < N; ++i) {
        if (i == without) continue;
        const Tile& t = tiles[i];
        const double groups = (double)(R < E ? R : E), mean = R / groups;
        const double blocks = E == 1 ? (double)((R + t.bm - 1) / t.bm) : mean <= 1.0 ? groups : groups * (mean / t.bm + 0.5 > 1.0 ? mean / t.bm + 0.5 : 1.0);
        const double per_cu = blocks * (double)((cols + t.bn - 1) / t.bn) / cus, x = per_cu / t.per_cu;
        const double rest = t.parts == 4 ? 0.28 : t.parts == 2 ? 0.32 : 0.5;
        double rounds = 1.0;
        if (E > 1) {
            rounds = x > 1.0 ? x + rest : x > 0.8 ? 1.0 + rest * (x - 0.8) / 0.2 : 1.0;   // (uneven groups may have more blocks)
        } else if (x > 1.0) {
            const int64_t whole = (int64_t)x;
            double last = x > whole ? 1.0 : 0.0;
            if (t.parts > 1 && x > whole) {
                const double split = (double)(int64_t)((x - whole) * t.parts + 0.999) * t.cost;
                if (split < 0.95) last = split;
            }
            rounds = whole + last;
        }
        const double alone = t.per_cu > 1 && x < 1.0 ? (x > 0.3 ? x : 0.3) : 1.0;   // where not every CU has all its items, each is done sooner
        const double time = rounds * (t.fixed + t.step * alone * (double)((bytes + 127) / 128));
        if (best < 0 || time < least) { best = i; least = time; }
    }
    return best;
}

}  // namespace ffuse
