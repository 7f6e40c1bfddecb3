// Matrix products grouped by expert: rows sorted by expert, a weight matrix for each.
//
//   forward : Y[r] = act(X[r] W[e]) [.* X[r] W3[e]]     X [R][K], W [E][K][N]
//   input   : dX[r] = dY[r] W[e]^T                       dY [R][N]
//   weights : dW[e] = X_e^T dY_e                         zeros for a group without rows
//
// The boundaries of the groups are on the device (ffuse_groups.h), so the host knows neither how many row blocks
// there are nor whose they are: forward and input run persistent workgroups, which each lay the row blocks of all
// groups end to end and take their share; a weight gradient's blocks are known beforehand.
#include "ffuse_gemm3.h"
#include "ffuse_groups.h"
#include "ffuse_launch.h"

namespace ffuse {

// ---- forward, and the gradient of the input -------------------------------------------------------------------------
// The rows of each group times its matrix, or its transpose: persistent workgroups; an item's first loads go out
// before the epilogue of the one before.  BCOL: Y = act(A W) (.* A W3), W [E][K][N]; otherwise Y = A W^T, W [E][N][K].
//
// 16384 rows in eight equal groups, and in eight uneven ones (68 row blocks for 64): gated 4096 x 11008 2249 and 2363 us
// (1.31 and 1.25 PFLOP/s), plain 11008 x 4096 1162 and 1262, 4096 x 4096 419 and 452, the gradient of the input 428 and 454.  Bound by the bytes from
// L2 to LDS and the power they take (the core clock is 1.9 - 2.1 GHz of 2.4): copies of the last without loads in the loop ran
// 358 us instead of 449, without fragment reads 433, with every workgroup of an XCD on the same panels 416.  A larger tile would move
// fewer bytes, but its accumulators do not fit.  512 rows of 64 experts, 1.1 GB of weights in two products: 186 us, 5.9 TB/s.
template <typename T, bool BCOL, bool GATED, class G, class Walk>
__device__ __forceinline__ void grouped_rows(const GroupedArgs& a, char* smem, Walk&& walk, int wave, int lane) {
    f32x4 acc[G::G][G::HT][G::MT];
    typename G::Ctx c;
    G::init(c, wave, lane);
    const int K = c.K = BCOL ? a.K : a.N, N = BCOL ? a.N : a.K;
    GroupItem it, next;
    bool have = walk.next(it), filled = false;
    auto aim = [&](const GroupItem& i) {
        c.a.aim(static_cast<const char*>(a.A) + i.row0 * K * 2, K, i.rows, K, wave, lane);
        const int64_t w = ((int64_t)i.e * K * N + (BCOL ? i.col : (int64_t)i.col * K)) * 2;
        c.b[0].aim(static_cast<const char*>(a.W) + w, BCOL ? N : K, N - i.col, K, wave, lane);
        if (GATED) c.b[G::G - 1].aim(static_cast<const char*>(a.W3) + w, BCOL ? N : K, N - i.col, K, wave, lane);
        G::fill(smem, c);
    };
    if (have) aim(it);
    while (have) {
        G::run(smem, c, acc, filled);
        have = walk.next(next);
        if (have) aim(next);
        filled = true;
        char* Y = static_cast<char*>(a.C) + (it.row0 * N + it.col) * 2;
        if (BCOL) G::store_rt(smem, a.act, acc, Y, (uint32_t)N, it.rows, N - it.col, wave);
        else G::template store<ACT_IDENTITY>(smem, acc, Y, (uint32_t)N, it.rows, N - it.col, wave);
        it = next;
    }
    // (the last steps' loads write to LDS, if only zeros: not after it is somebody else's)
    lds_loads_in_flight_at_most<0>();
}

// G: the tile of an item; S: of its parts (whole_items), `cost` of it each, or G itself
template <typename T, bool BCOL, bool GATED, class G, class S>
__global__ __launch_bounds__(64 * G::NW) void grouped_rows_kernel(GroupedArgs a, float cost) {
    constexpr int PARTS = (G::BM / S::BM) * (G::BN / S::BN), LDS = G::LDS_BYTES > S::LDS_BYTES ? G::LDS_BYTES : S::LDS_BYTES;
    static_assert(LDS <= kLdsBesideGroups, "LDS");
    static_assert(G::NW == S::NW, "one workgroup does both");
    __shared__ __attribute__((aligned(16))) char smem[LDS];
    extern __shared__ __attribute__((aligned(16))) char table[];
    const int tid = threadIdx.x, xcd = blockIdx.x & 7, loc = blockIdx.x >> 3, step = gridDim.x >> 3, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    Groups groups;
    scan_groups(groups, table, smem, a.offsets, a.E, a.R, G::BM, tid);
    const int N = BCOL ? a.N : a.K, ncol = (N + G::BN - 1) / G::BN;
    const int items = group_items(groups, ncol, xcd), whole = PARTS > 1 ? whole_items<PARTS>(items, step, cost) : items;
    grouped_rows<T, BCOL, GATED, G>(a, smem, ItemWalk<G::BM, G::BN, 1>{groups, G::BM, G::BN, ncol, N, xcd, 0, whole, step, loc}, wave, lane);
    if constexpr (PARTS > 1) {
        if (whole < items) {
            __syncthreads();
            grouped_rows<T, BCOL, GATED, S>(a, smem, ItemWalk<S::BM, S::BN, PARTS>{groups, G::BM, G::BN, ncol, N, xcd, whole, items - whole, step, loc}, wave, lane);
        }
    }
}

// ---- gradient of the weights ------------------------------------------------------------------------------------
// One block of one group's gradient a workgroup, in order of the groups: the hardware hands them out as CUs come
// free, which evens out groups of different lengths.  16384 rows, 4096 x 4096: 467 us, 1.18 PFLOP/s, in equal and in uneven groups alike (copies without
// loads in the loop 383, without fragment reads 440 -- both operands go through transposing reads, two for one).  Persistent
// workgroups with equal shares and early first loads took 517.
template <typename T, int BM, int BN, int WM, int WN, int NS>
__global__ __launch_bounds__(64 * WM * WN) void grouped_weights_kernel(GroupedArgs a) {
    typedef PairGemm<T, true, true, false, BM, BN, WM, WN, NS> G;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int mb = (a.K + BM - 1) / BM, nb = (a.N + BN - 1) / BN;
    const int e = (int)(blockIdx.x / (uint32_t)(mb * nb)), b = (int)(blockIdx.x % (uint32_t)(mb * nb));
    // (any boundaries are taken: the rows read are inside the tensor, and nothing but dW[e] is written)
    const int first = min(max(a.offsets[e], 0), a.R), last = min(max(a.offsets[e + 1], 0), a.R);
    const int band = b / (kGroupBand * nb), in = b - band * kGroupBand * nb, h = min(kGroupBand, mb - band * kGroupBand);
    const int m0 = (band * kGroupBand + in % h) * BM, n0 = in / h * BN;
    f32x4 acc[G::G][G::HT][G::MT];
    typename G::Ctx c;
    G::init(c, wave, lane);
    c.K = max(last - first, 0);
    c.a.aim(static_cast<const char*>(a.A) + ((int64_t)first * a.K + m0) * 2, a.K, a.K - m0, c.K, wave, lane);
    c.b[0].aim(static_cast<const char*>(a.W) + ((int64_t)first * a.N + n0) * 2, a.N, a.N - n0, c.K, wave, lane);
    G::fill(smem, c);
    G::run(smem, c, acc, false);
    lds_loads_in_flight_at_most<0>();   // (loads past the last stage write to LDS, if only zeros: not after the workgroup is gone)
    char* dW = static_cast<char*>(a.C) + ((int64_t)e * a.K * a.N + (int64_t)m0 * a.N + n0) * 2;
    G::template store<ACT_IDENTITY>(smem, acc, dW, (uint32_t)a.N, a.K - m0, a.N - n0, wave);
}

// ---- launches ---------------------------------------------------------------------------------------------------
// Tiles, and their times for 64 k, set on 16384 rows in eight uneven groups (4096 x 11008 gated, 11008 x 4096 plain, 4096 x 4096 for
// the gradient of the input, whose operands need no transposing) and on 160 drawn problems of 1 to 16384 rows and 1 to 128
// groups for each of the three tables, every tile timed on each: what is chosen takes 2 % more time than the best of them on average.  128 x 128, where
// there are too few blocks of 128 x 256 for the CUs: 568 rows in five groups, 7168 x 3336, 75 us instead of 97 (plain) and 68
// instead of 93 (input); 3184 in 23, 11656 x 576, 132 instead of 154 and 178 instead of 231.  A wave's part is 128 x 64 of the
// largest (256 x 128 gated: 128 x 32 of either branch) and 32 x 32 of the small ones.
static constexpr Tile kGated[] = {{256, 128, 1, 1.60f, 2.0f, 4, 0.36f}, {128, 128, 1, 1.00f, 2.0f, 2, 0.76f}, {64, 128, 1, 0.68f, 2.0f, 1, 1.0f},
                                  {32, 128, 1, 0.58f, 2.0f, 1, 1.0f}, {64, 64, 2, 1.15f, 2.0f, 1, 1.0f}};
static constexpr Tile kPlain[] = {{256, 256, 1, 1.59f, 2.0f, 4, 0.38f}, {128, 256, 1, 0.97f, 2.0f, 4, 0.46f}, {128, 128, 1, 0.60f, 2.0f, 2, 0.73f},
                                  {64, 256, 1, 0.67f, 2.0f, 2, 0.64f},  {64, 128, 1, 0.44f, 2.0f, 1, 1.0f},   {32, 128, 1, 0.37f, 2.0f, 1, 1.0f},
                                  {64, 64, 2, 0.72f, 2.0f, 1, 1.0f}};
static constexpr Tile kInput[] = {{256, 256, 1, 1.50f, 2.0f, 4, 0.38f}, {128, 256, 1, 0.94f, 2.0f, 4, 0.46f}, {128, 128, 1, 0.59f, 2.0f, 2, 0.64f},
                                  {64, 256, 1, 0.63f, 2.0f, 2, 0.64f},  {64, 128, 1, 0.36f, 2.0f, 1, 1.0f},   {32, 128, 1, 0.27f, 2.0f, 1, 1.0f},
                                  {64, 64, 2, 0.66f, 2.0f, 1, 1.0f}};

template <typename T, bool BCOL, bool GATED, class G, class S> static hipError_t rows(const GroupedArgs& a, const Tile& t, int cus, hipStream_t st) {
    const int N = BCOL ? a.N : a.K;
    const int grid = persistent_grid(most_row_blocks(a.R, a.E, G::BM) * ((N + G::BN - 1) / G::BN), cus, t.per_cu);
    hipLaunchKernelGGL((grouped_rows_kernel<T, BCOL, GATED, G, S>), dim3(grid), dim3(64 * G::NW), group_table_bytes(a.E), st, a, t.cost);
    return hipGetLastError();
}
template <typename T> static hipError_t gated(const GroupedArgs& a, int cus, hipStream_t st) {
    typedef PairGemm<T, false, true, true, 256, 128, 2, 4, 2> G256;
    typedef PairGemm<T, false, true, true, 128, 64, 4, 2, 4> Q256;
    typedef PairGemm<T, false, true, true, 128, 128, 2, 4, 3> G128;
    typedef PairGemm<T, false, true, true, 64, 128, 2, 4, 3> G64;
    typedef PairGemm<T, false, true, true, 32, 128, 1, 4, 3> G32;
    typedef PairGemm<T, false, true, true, 64, 64, 2, 2, 3> S64;
    // The last tile's tables leave room for one workgroup a CU where there are more than 512 groups: it is only taken where one is all
    // that a CU gets.  us, as for two a CU -> this: 125 rows in 813 groups, 416 x 176, 29.2 -> 17.6; 34218 in 1018, 560 x 64, 63.2 -> 48.8.
    // (Never above 512 groups: 65 rows in 839, 1776 x 64, 24.8 -> 26.8.)
    const bool alone = a.E > most_groups(S64::LDS_BYTES, kGated[4].per_cu);
    const bool full = most_row_blocks(a.R, a.E, S64::BM) * ((a.N + S64::BN - 1) / S64::BN) > cus;
    const int i = pick_tile(kGated, a.R, a.E, a.N, 2 * (int64_t)a.K, cus, alone && full ? 4 : -1);
    switch (i) {
        case 0: return rows<T, true, true, G256, Q256>(a, kGated[i], cus, st);
        case 1: return rows<T, true, true, G128, G64>(a, kGated[i], cus, st);
        case 2: return rows<T, true, true, G64, G64>(a, kGated[i], cus, st);
        case 3: return rows<T, true, true, G32, G32>(a, kGated[i], cus, st);
        default: return rows<T, true, true, S64, S64>(a, kGated[i], cus, st);
    }
}
template <typename T, bool BCOL> static hipError_t plain(const GroupedArgs& a, int cus, hipStream_t st) {
    typedef PairGemm<T, false, BCOL, false, 256, 256, 2, 4, 2> G256;
    typedef PairGemm<T, false, BCOL, false, 128, 256, 2, 4, 3> W128;
    typedef PairGemm<T, false, BCOL, false, 128, 128, 2, 4, 4> G128;
    typedef PairGemm<T, false, BCOL, false, 64, 256, 2, 4, 3> W64;
    typedef PairGemm<T, false, BCOL, false, 64, 128, 2, 4, 4> G64;
    typedef PairGemm<T, false, BCOL, false, 32, 128, 1, 4, 4> G32;
    typedef PairGemm<T, false, BCOL, false, 64, 64, 2, 2, 4> S64;
    static_assert(most_groups(S64::LDS_BYTES, kPlain[6].per_cu) >= kMaxGroups && kInput[6].per_cu == kPlain[6].per_cu, "two workgroups a CU");
    const int i = BCOL ? pick_tile(kPlain, a.R, a.E, a.N, 2 * (int64_t)a.K, cus) : pick_tile(kInput, a.R, a.E, a.K, 2 * (int64_t)a.N, cus);
    const Tile& t = BCOL ? kPlain[i] : kInput[i];
    switch (i) {
        case 0: return rows<T, BCOL, false, G256, G128>(a, t, cus, st);
        case 1: return rows<T, BCOL, false, W128, G64>(a, t, cus, st);
        case 2: return rows<T, BCOL, false, G128, G64>(a, t, cus, st);
        case 3: return rows<T, BCOL, false, W64, G64>(a, t, cus, st);
        case 4: return rows<T, BCOL, false, G64, G64>(a, t, cus, st);
        case 5: return rows<T, BCOL, false, G32, G32>(a, t, cus, st);
        default: return rows<T, BCOL, false, S64, S64>(a, t, cus, st);
    }
}
hipError_t launch_grouped_forward(int dtype, const GroupedArgs& a, int cus, hipStream_t st) {
    if (a.W3) return dtype == 0 ? gated<__bf16>(a, cus, st) : gated<_Float16>(a, cus, st);
    return dtype == 0 ? plain<__bf16, true>(a, cus, st) : plain<_Float16, true>(a, cus, st);
}
hipError_t launch_grouped_input(int dtype, const GroupedArgs& a, int cus, hipStream_t st) {
    return dtype == 0 ? plain<__bf16, false>(a, cus, st) : plain<_Float16, false>(a, cus, st);
}

template <typename T, int BM, int BN, int WM, int WN, int NS> static hipError_t weights(const GroupedArgs& a, hipStream_t st) {
    const int64_t grid = (int64_t)a.E * ((a.K + BM - 1) / BM) * ((a.N + BN - 1) / BN);
    hipLaunchKernelGGL((grouped_weights_kernel<T, BM, BN, WM, WN, NS>), dim3((unsigned)grid), dim3(64 * WM * WN), 0, st, a);
    return hipGetLastError();
}
// 256 x 256 takes 1.9 us for 64 rows, two of 128 x 128 side by side 1.2: four fill as many CUs twice as well, where there are few.
// (Times of long groups.  The 4 us beside them are the same for both, though the larger tile stores four times as much, and with few rows
// a group the rule is off: 1501 rows in 12 groups, 1000 x 1352, 19 us where it expects 11.)
template <typename T> static hipError_t weights_any(const GroupedArgs& a, int cus, hipStream_t st) {
    const auto items = [&](int b) { return (double)a.E * ((a.K + b - 1) / b) * ((a.N + b - 1) / b); };
    const double steps = (double)a.R / a.E / 64, big = items(256) / cus, small = items(128) / (2 * cus);
    const double t_big = (big <= 1.0 ? 1.0 : big + 0.3) * (4.0 + 1.9 * steps);
    const double t_small = (small <= 1.0 ? 1.0 : small + 0.3) * (4.0 + 1.2 * (small <= 0.5 ? 0.6 : 1.0) * steps);
    if (t_big <= t_small) return weights<T, 256, 256, 2, 4, 2>(a, st);
    return weights<T, 128, 128, 2, 2, 2>(a, st);
}
hipError_t launch_grouped_weights(int dtype, const GroupedArgs& a, int cus, hipStream_t st) {
    return dtype == 0 ? weights_any<__bf16>(a, cus, st) : weights_any<_Float16>(a, cus, st);
}

}  // namespace ffuse
