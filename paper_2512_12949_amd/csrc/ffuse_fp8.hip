// Products in 8-bit floating point (e4m3) with a scale for each block of 128 along the contraction, dense or grouped
// by expert, and the pass that quantises their operands.
//
//   Y[m][n] = sum over blocks b of  sa[b][m] sb[b][n / block] * sum over k in b of  A[m][k] B[n][k]
//
// Both operands are contiguous along k.  A block's products are summed by ONE matrix instruction
// (16 x 16 outputs, 128 k), exactly that sum is multiplied with sa sb, which may be any fp32 numbers, and added to
// the fp32 accumulators: one multiply-add per output and block beside the matrix pipe's 8 passes.
// (What the instruction itself keeps: it aligns the products of eight neighbouring k with the largest of the eight and drops
// what lies more than 13 binary places below that one's leading bit; the groups' sums are added in fp32.)
#include "ffuse_gemm3.h"
#include "ffuse_groups.h"
#include "ffuse_launch.h"

namespace ffuse {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;

// D[16][16] += A[16][128] B[16][128]^T: lane l holds 32 bytes of row l % 16 of either operand, the same 32 k of both, and of D
// column l % 16, rows 4 (l / 16) + r.
__device__ __forceinline__ f32x4 mma_e4m3(i32x8 a, i32x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
}

// 4 bytes a lane to LDS bytes [lds, lds + 256)
__device__ __forceinline__ void lds_load4(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\tbuffer_load_dword %0, %2, 0 offen lds" :: "v"(voff), "s"(lds), "s"(r) : "memory", "m0");
}

// A stage is 128 k: BM + BN rows of 128 bytes, laid out as PairOperand lays out rows that are contiguous along the contraction, and
// behind them their BM + BN scales of that block.
// Computed transposed like the other block GEMMs: the MFMA "A" operand is B, so that a lane has four neighbouring
// columns of one row of Y.
//
// A step multiplies one stage, 16 rows after 16 rows: the fragments of the wave's columns stay in registers, those of a row
// block are read two blocks ahead, and beside each MFMA run the multiply-adds of the one four before it.  The workgroup meets before
// the last two row blocks, whose fragments are in registers by then: the next stage has landed, and the present one is free
// for the loads of the stage NS further on.  Those two go through the columns together, so that a column's fragment is free for
// the next step's after two products and its reads spread over eight.  (One row block behind the barrier, read one block
// ahead: 4096 x 4096 x 16384 in 247 us instead of 237.)
//
// What bounds it: 2.3 PFLOP/s at that size, the matrix pipes busy half of the time.  A copy of the kernel without loads in
// the loop took 208 us instead of 240, one without fragment reads 242: the bytes from L2 to LDS, not LDS itself.
// (256 x 256 takes all 256 registers; with scales of single columns four more, which are spilled outside the loop and reloaded
// once an item.)
template <typename T, int BM_, int BN_, int WM, int WN, int NS, int BLOCK_> struct Fp8Gemm {
    static constexpr int BM = BM_, BN = BN_, BLOCK = BLOCK_, NW = WM * WN, WMR = BM / WM, WNR = BN / WN, MT = WMR / 16, HT = WNR / 16;
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "every wave issues the same number of loads");
    static_assert(BLOCK == 1 || BLOCK == 128, "scales of B");
    static_assert(128 % WNR == 0, "a wave's columns share a block of 128");
    static constexpr int XI = BM / 8 / NW, BI = BN / 8 / NW;
    static constexpr int SA = (BM + 63) / 64, SB = (BN + 63) / 64;        // scale load instructions of a stage: 64 rows each
    static constexpr int SI = (SA + SB + NW - 1) / NW;                    // ... per wave (some are issued twice)
    static constexpr int NLOAD = XI + BI + SI;
    static constexpr int XB = BM * 128, SOFF = XB + BN * 128, STAGE = SOFF + (SA + SB) * 256;
    // (a wave's columns leave 32 at a time where the ring leaves no room for 64)
    static constexpr int ECOL = WNR == 64 && NS * STAGE + NW * 2048 > 152 * 1024 ? 32 : WNR;
    typedef TileStore<T, ECOL, MT> Store;
    static constexpr int EPI = NS * STAGE, LDS_BYTES = EPI + NW * Store::LDS_BYTES, STORES = WNR / ECOL * MT * Store::STORES;
    static_assert(NS >= 2 && (NS - 1) * NLOAD + STORES <= 63, "the vmcnt field holds 6 bits");
    static_assert(MT % 2 == 0, "the last rows' fragments and the next step's first lie in different registers");
    static constexpr int NM = MT * HT, LAG = HT < 4 ? HT : 4;             // MFMAs a step; parts in flight

    struct Ctx {
        __amdgpu_buffer_rsrc_t rx, rw;
        const float *sa, *sb;          // block 0's scales of the tile's first row / of B's first column
        int64_t sa_step, sb_step;      // floats from block to block
        uint32_t have_a, have_b;       // bytes of the tile's scales (of a block)
        uint32_t xoff[XI], boff[BI], soff[SI];
        int ck, K;
        uint32_t lds_a, lds_b;
        uint32_t rdx, rdw;             // this lane's first row of either operand in a stage (16 rows on: 2048 bytes, the same swizzle)
        uint32_t sx;                   // LDS offset of this lane's row scale in a stage
        uint32_t sw;                   // ... of its first column scale
    };
    template <int N> static __device__ __forceinline__ void rows(uint32_t (&off)[N], int have, int K, int tid) {
        const int wave = tid >> 6, lane = tid & 63;
        const uint32_t chunk = (lane & 7u) ^ (uint32_t)(((wave & 1) << 2) | (lane >> 4));
#pragma unroll
        for (int j = 0; j < N; ++j) off[j] = (uint32_t)min(8 * (wave + NW * j) + (lane >> 3), have - 1) * (uint32_t)K + 16u * chunk;
    }
    static __device__ __forceinline__ void init_lds(Ctx& c, int tid) {
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
        const int wm = wave % WM, wn = wave / WM;
        const uint32_t x = lane & 15, g = lane >> 4;
        c.ck = 16 * ((lane & 7) ^ (((wave & 1) << 2) | (lane >> 4)));
        c.lds_a = (uint32_t)wave * 1024u;
        c.lds_b = XB + (uint32_t)wave * 1024u;
        c.rdx = (wm * WMR + x) * 128u + ((g ^ ((x >> 1) & 7u)) << 4);
        c.rdw = XB + (wn * WNR + x) * 128u + ((g ^ ((x >> 1) & 7u)) << 4);
        c.sx = SOFF + 4u * (uint32_t)(wm * WMR + x);
        c.sw = SOFF + SA * 256u + 4u * (uint32_t)(wn * WNR + (BLOCK == 1 ? 4 * g : 0));
    }
    // A: the tile's first row, B: the tile's first column's row
    static __device__ __forceinline__ void aim(Ctx& c, const char* A, const float* sa, int64_t sa_step, int have_a,
                                               const char* B, const float* sb, int64_t sb_step, int have_b, int K, int tid) {
        have_a = min(have_a, BM); have_b = min(have_b, BN);
        c.rx = make_rsrc(A, (uint32_t)have_a * (uint32_t)K);
        c.rw = make_rsrc(B, (uint32_t)have_b * (uint32_t)K);
        c.K = K;
        rows<XI>(c.xoff, have_a, K, tid);
        rows<BI>(c.boff, have_b, K, tid);
        c.sa = sa; c.sb = sb; c.sa_step = sa_step; c.sb_step = sb_step;
        c.have_a = 4u * (uint32_t)have_a; c.have_b = 4u * (uint32_t)((have_b + BLOCK - 1) / BLOCK);
        const int wave = tid >> 6, lane = tid & 63;
#pragma unroll
        for (int j = 0; j < SI; ++j) {
            const int i = (wave * SI + j) % (SA + SB);
            c.soff[j] = 4u * (uint32_t)(i < SA ? min(64 * i + lane, have_a - 1) : min(64 * (i - SA) + lane, have_b - 1) / BLOCK);
        }
    }
    // Load i of the stage of block b.  One past the last is issued all the same, out of range: it fetches nothing and writes zeros
    // to a place that nobody reads, and every step has the same number of loads in flight.
    static __device__ __forceinline__ void issue_one(const Ctx& c, uint32_t stage, int b, int i, int wave) {
        const uint32_t k = 128u * (uint32_t)b;
        if (i < XI) lds_load16(c.rx, 128 * b + c.ck < c.K ? c.xoff[i] + k : kOob, stage + c.lds_a + (uint32_t)(i * NW) * 1024u);
        else if (i < XI + BI) lds_load16(c.rw, 128 * b + c.ck < c.K ? c.boff[i - XI] + k : kOob, stage + c.lds_b + (uint32_t)((i - XI) * NW) * 1024u);
        else {
            const int j = i - XI - BI, n = (wave * SI + j) % (SA + SB);
            const bool ok = 128 * b < c.K;
            const __amdgpu_buffer_rsrc_t r = n < SA ? make_rsrc(c.sa + b * c.sa_step, ok ? c.have_a : 0u) : make_rsrc(c.sb + b * c.sb_step, ok ? c.have_b : 0u);
            lds_load4(r, c.soff[j], stage + SOFF + 256u * (uint32_t)n);
        }
    }
    // the loads of an item's first NS stages
    static __device__ __forceinline__ void fill(char* smem, const Ctx& c, int wave) {
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int i = 0; i < NLOAD; ++i) issue_one(c, (uint32_t)(uintptr_t)smem + (uint32_t)(j * STAGE), j, i, wave);
    }
    static __device__ __forceinline__ i32x8 frag(const char* p, const char* q) {
        const i32x4 lo = __builtin_bit_cast(i32x4, *reinterpret_cast<const u32x4*>(p)), hi = __builtin_bit_cast(i32x4, *reinterpret_cast<const u32x4*>(q));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    struct Frags {
        i32x8 a[HT], b[4];   // the columns' fragments; those of the last row blocks read
        float s[4];          // and their rows' scales
    };
    static __device__ __forceinline__ void read_a(const char* stage, const Ctx& c, Frags& f, int ht) {
        f.a[ht] = frag(stage + c.rdw + 2048 * ht, stage + (c.rdw ^ 64u) + 2048 * ht);
    }
    static __device__ __forceinline__ void read_b(const char* stage, const Ctx& c, Frags& f, int mt, int place) {
        f.b[place] = frag(stage + c.rdx + 2048 * mt, stage + (c.rdx ^ 64u) + 2048 * mt);
        f.s[place] = *reinterpret_cast<const float*>(stage + c.sx + 64 * mt);
    }
    // filled: the first stages were issued before the epilogue of the item before, whose stores are younger
    static __device__ __forceinline__ void run(char* smem, const Ctx& c, f32x4 (&acc)[HT][MT], int wave, bool filled) {
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ht = 0; ht < HT; ++ht)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc[ht][mt] = zero;
        const int KT = (c.K + 127) / 128;
        const uint32_t lds = (uint32_t)(uintptr_t)smem;
        if (filled) lds_loads_in_flight_at_most<(NS - 1) * NLOAD + STORES>();
        else lds_loads_in_flight_at_most<(NS - 1) * NLOAD>();
        __syncthreads();
        Frags f;
        f32x4 part[LAG];
        read_b(smem, c, f, 0, 0);
#pragma unroll
        for (int ht = 0; ht < HT; ++ht) read_a(smem, c, f, ht);
        read_b(smem, c, f, 1, 1);
        constexpr int FIRST = MT % 4 ? 2 : 0;   // where the next step's first row blocks are read to
        int slot = 0;
        for (int s = 0; s < KT; ++s) {
            const char* cur = smem + slot * STAGE;
            const uint32_t ld = lds + (uint32_t)(slot * STAGE);
            slot = slot == NS - 1 ? 0 : slot + 1;
            const char* nxt = smem + slot * STAGE;
            // the columns' scales, first used LAG products on
            f32x4 sw[BLOCK == 1 ? HT : 1];
            float sw0 = 1.0f, row[4];
            if (BLOCK == 1) {
#pragma unroll
                for (int ht = 0; ht < (BLOCK == 1 ? HT : 1); ++ht) sw[ht] = *reinterpret_cast<const f32x4*>(cur + c.sw + 64 * ht);
            } else {
                sw0 = *reinterpret_cast<const float*>(cur + c.sw);
            }
            // MFMA i: row block mt, columns ht; the last two row blocks go through the columns together
            constexpr int JOINT = NM - 2 * HT;
            auto mt_of = [](int i) { return i < JOINT ? i / HT : MT - 2 + ((i - JOINT) & 1); };
            auto ht_of = [](int i) { return i < JOINT ? i % HT : (i - JOINT) / 2; };
            auto add = [&](int j) {
                const int mt = mt_of(j), ht = ht_of(j);
                if (ht == 0) row[mt & 3] = BLOCK == 1 ? f.s[mt & 3] : f.s[mt & 3] * sw0;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    acc[ht][mt][r] = __builtin_fmaf(part[j % LAG][r], BLOCK == 1 ? sw[BLOCK == 1 ? ht : 0][r] * row[mt & 3] : row[mt & 3], acc[ht][mt][r]);
            };
#pragma unroll
            for (int i = 0; i < NM; ++i) {
                const int mt = mt_of(i), ht = ht_of(i);
                if (i >= LAG) add(i - LAG);
                if (ht == 0 && mt + 2 < MT) read_b(cur, c, f, mt + 2, (mt + 2) & 3);
                if (i == JOINT) {
                    lds_loads_in_flight_at_most<(NS - 2) * NLOAD>();
                    __syncthreads();
                }
                part[i % LAG] = mma_e4m3(f.a[ht], f.b[mt & 3], zero);
                if (i >= JOINT) {
                    const int p = i - JOINT;
                    if (p & 1) read_a(nxt, c, f, ht);
                    else if (p < 4) read_b(nxt, c, f, p / 2, FIRST + p / 2);
#pragma unroll
                    for (int e = p * NLOAD / (2 * HT); e < (p + 1) * NLOAD / (2 * HT); ++e) issue_one(c, ld, s + NS, e, wave);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int j = NM - LAG; j < NM; ++j) add(j);
            if (FIRST) {
#pragma unroll
                for (int j = 0; j < 2; ++j) { f.b[j] = f.b[FIRST + j]; f.s[j] = f.s[FIRST + j]; }
            }
        }
        __syncthreads();   // the stages are the next item's
    }
    // Y: the tile's first row and column
    static __device__ __forceinline__ void store(char* smem, const f32x4 (&acc)[HT][MT], char* Y, uint32_t ldy, int have_m, int have_n, int wave) {
#pragma unroll
        for (int e = 0; e < WNR / ECOL; ++e)
            Store::store(smem + EPI + wave * Store::LDS_BYTES, Y, ldy, wave % WM * WMR, wave / WM * WNR + e * ECOL, BM, have_m, have_n,
                         [&](int h, int mt, int r) { return acc[e * (ECOL / 16) + h][mt][r]; });
    }
};

// LDS of the largest tile, which leaves room for the tables of kFp8Groups groups
static constexpr int kFp8Lds = 160256, kFp8Groups = (160 * 1024 - kFp8Lds) / 8;
static_assert(group_table_bytes(kFp8Groups) <= 160 * 1024 - kFp8Lds, "LDS");

template <class G, class Walk> __device__ __forceinline__ void fp8_rows(const Fp8Args& a, char* smem, Walk&& walk, int tid, int wave) {
    f32x4 acc[G::HT][G::MT];
    typename G::Ctx c;
    G::init_lds(c, tid);
    const int KB = (a.K + 127) / 128, NB = (a.N + G::BLOCK - 1) / G::BLOCK;
    GroupItem it, next;
    bool have = walk.next(it), filled = false;
    auto aim = [&](const GroupItem& i) {
        G::aim(c, static_cast<const char*>(a.A) + i.row0 * a.K, a.sa + i.row0, a.R, i.rows,
               static_cast<const char*>(a.B) + ((int64_t)i.e * a.N + i.col) * a.K, a.sb + (int64_t)i.e * KB * NB + i.col / G::BLOCK, NB, a.N - i.col, a.K, tid);
        G::fill(smem, c, wave);
    };
    if (have) aim(it);
    while (have) {
        G::run(smem, c, acc, wave, filled);
        have = walk.next(next);
        if (have) aim(next);
        filled = true;
        G::store(smem, acc, static_cast<char*>(a.Y) + (it.row0 * a.N + it.col) * 2, (uint32_t)a.N, it.rows, a.N - it.col, wave);
        it = next;
    }
    // (the last steps' loads write to LDS, if only zeros: not after it is somebody else's)
    lds_loads_in_flight_at_most<0>();
}
// G: the tile of an item; S: of its parts (whole_items), `cost` of it each, or G itself
template <class G, class S> __global__ __launch_bounds__(64 * G::NW) void fp8_product_kernel(Fp8Args a, float cost) {
    constexpr int PARTS = (G::BM / S::BM) * (G::BN / S::BN), LDS = G::LDS_BYTES > S::LDS_BYTES ? G::LDS_BYTES : S::LDS_BYTES;
    static_assert(LDS <= kFp8Lds, "LDS");
    static_assert(G::NW == S::NW, "one workgroup does both");
    __shared__ __attribute__((aligned(16))) char smem[LDS];
    extern __shared__ __attribute__((aligned(16))) char table[];
    const int tid = threadIdx.x, xcd = blockIdx.x & 7, loc = blockIdx.x >> 3, step = gridDim.x >> 3, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    Groups groups;
    scan_groups(groups, table, smem, a.offsets, a.E, a.R, G::BM, tid);
    const int ncol = (a.N + G::BN - 1) / G::BN;
    const int items = group_items(groups, ncol, xcd), whole = PARTS > 1 ? whole_items<PARTS>(items, step, cost) : items;
    fp8_rows<G>(a, smem, ItemWalk<G::BM, G::BN, 1>{groups, G::BM, G::BN, ncol, a.N, xcd, 0, whole, step, loc}, tid, wave);
    if constexpr (PARTS > 1) {
        if (whole < items) {
            __syncthreads();
            fp8_rows<S>(a, smem, ItemWalk<S::BM, S::BN, PARTS>{groups, G::BM, G::BN, ncol, a.N, xcd, whole, items - whole, step, loc}, tid, wave);
        }
    }
}

// Few rows: the weights' way from memory is all that counts.  A workgroup has 16 columns and 16 MT rows, its eight waves every
// eighth block of 128 k each, and a wave two blocks in flight, straight from memory to the registers of the matrix
// instruction (16 rows of B x 128 bytes, whole cache lines, are its operand as they lie); the waves' sums meet in LDS, in
// their order.  One row of 4096 x 11008 in 12.2 us, 3.7 TB/s: 3 us of it are the launch and the first loads' way.
template <typename T, int MT, int BLOCK> __global__ __launch_bounds__(512) void fp8_stream_kernel(Fp8Args a) {
    constexpr int NW = 8, DEPTH = 2;
    __shared__ __attribute__((aligned(16))) f32x4 sums[NW][MT][64];
    extern __shared__ __attribute__((aligned(16))) char table[];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const uint32_t x = lane & 15, g = lane >> 4;
    GroupItem it;
    const int ncol = (a.N + 15) / 16, KB = (a.K + 127) / 128, NB = (a.N + BLOCK - 1) / BLOCK;
    if (a.offsets) {
        Groups groups;
        scan_groups(groups, table, reinterpret_cast<char*>(sums), a.offsets, a.E, a.R, 16 * MT, tid);
        const int xcd = blockIdx.x & 7, idx = blockIdx.x >> 3;
        if (idx >= group_items(groups, ncol, xcd)) return;
        it = group_item(groups, 16 * MT, 16, ncol, xcd, idx);
    } else {
        it.e = 0;
        it.row0 = (int64_t)(blockIdx.x / (uint32_t)ncol) * (16 * MT);
        if (it.row0 >= a.R) return;
        it.rows = a.R - (int)it.row0;
        it.col = 16 * (int)(blockIdx.x % (uint32_t)ncol);
    }
    const int n0 = it.col, rows = min(it.rows, 16 * MT), cols = min(a.N - n0, 16);
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(static_cast<const char*>(a.A) + it.row0 * a.K, (uint32_t)rows * (uint32_t)a.K);
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(static_cast<const char*>(a.B) + ((int64_t)it.e * a.N + n0) * a.K, (uint32_t)cols * (uint32_t)a.K);
    const float* sa = a.sa + it.row0;
    const float* sb = a.sb + (int64_t)it.e * KB * NB + n0 / BLOCK;
    uint32_t xo[MT], so[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const uint32_t row = (uint32_t)min(16 * mt + (int)x, rows - 1);
        xo[mt] = row * (uint32_t)a.K + 16u * g;
        so[mt] = 4u * row;
    }
    const uint32_t wo = (uint32_t)min((int)x, cols - 1) * (uint32_t)a.K + 16u * g;
    const uint32_t bo = BLOCK == 1 ? 16u * min(g, (uint32_t)(cols - 1) / 4u) : 0u;   // (columns come in eights)
    struct Slot {
        u32x4 w[2], x[MT][2];
        f32x4 sw;
        float sx[MT];
    } t[DEPTH];
    auto load = [&](Slot& d, int kb) {
        const uint32_t k = 128u * (uint32_t)kb;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bool ok = 128 * kb + 64 * h + 16 * (int)g < a.K;
            d.w[h] = buf_load16(rw, ok ? wo + k + 64u * h : kOob);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) d.x[mt][h] = buf_load16(rx, ok ? xo[mt] + k + 64u * h : kOob);
        }
        const bool ok = kb < KB;
        const __amdgpu_buffer_rsrc_t ra = make_rsrc(sa + (int64_t)kb * a.R, ok ? 4u * (uint32_t)rows : 0u);
        const __amdgpu_buffer_rsrc_t rb = make_rsrc(sb + (int64_t)kb * NB, ok ? 4u * (uint32_t)(BLOCK == 1 ? cols : 1) : 0u);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) d.sx[mt] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(ra, so[mt], 0, 0));
        if (BLOCK == 1) d.sw = __builtin_bit_cast(f32x4, buf_load16(rb, bo));
        else d.sw[0] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rb, 0, 0, 0));
    };
    f32x4 acc[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](const Slot& d) {
        const i32x8 w = __builtin_shufflevector(__builtin_bit_cast(i32x4, d.w[0]), __builtin_bit_cast(i32x4, d.w[1]), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const i32x8 r = __builtin_shufflevector(__builtin_bit_cast(i32x4, d.x[mt][0]), __builtin_bit_cast(i32x4, d.x[mt][1]), 0, 1, 2, 3, 4, 5, 6, 7);
            const f32x4 part = mma_e4m3(w, r, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[mt][e] = __builtin_fmaf(part[e], d.sx[mt] * d.sw[BLOCK == 1 ? e : 0], acc[mt][e]);
        }
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) load(t[d], wave + NW * d);
    for (int kb = wave; kb < KB; kb += NW * DEPTH)
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            multiply(t[d]);
            __builtin_amdgcn_sched_barrier(0);
            load(t[d], kb + NW * (d + DEPTH));
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) sums[wave][mt][lane] = acc[mt];
    __syncthreads();
    if (wave >= MT) return;
    f32x4 y = sums[0][wave][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) y += sums[w][wave][lane];
    const int m = 16 * wave + (int)x, n = 4 * (int)g;
    if (m < rows && n < cols)
        *reinterpret_cast<uint2*>(static_cast<char*>(a.Y) + ((it.row0 + m) * a.N + n0 + n) * 2) = uint2{pack2<T>(y[0], y[1]), pack2<T>(y[2], y[3])};
}

// ---- quantising -------------------------------------------------------------------------------------------------
// The scale of a block: the smallest power of two that brings its largest finite magnitude to 448, e4m3's largest number,
// or below -- 2^(e - 8) for a magnitude of 2^e (1 .. 1.75), 2^(e - 7) above; 2^-126 at least; 1 for a block of
// zeros.  Dividing by it is exact (it only moves the exponent), so the one rounding is the one to e4m3, to nearest even.
// Infinities and NaN do not count for the scale and are stored as NaN.
__device__ __forceinline__ uint32_t finite_magnitude(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
    return b >= 0x7f800000u ? 0u : b;
}
__device__ __forceinline__ float block_scale(uint32_t largest) {
    if (largest == 0u) return 1.0f;
    const int e = (int)((largest + 0x1fffffu) >> 23);      // the exponent field, one more where the fraction passes 0.75
    return __builtin_bit_cast(float, (uint32_t)max(e - 8, 1) << 23);
}
__device__ __forceinline__ float inverse_of_power(float scale) { return __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(uint32_t, scale)); }
// four neighbouring values, scaled, as e4m3
__device__ __forceinline__ uint32_t to_e4m3(const float* v, float inv) {
    float s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = (v[i] - v[i] == 0.0f) ? v[i] * inv : __builtin_nanf("");
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(s[0], s[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(s[2], s[3], w, true);
}
template <typename T> __device__ __forceinline__ void widen8(u32x4 w, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2<T>(w[i], v[2 * i], v[2 * i + 1]);
}

struct QuantArgs {
    const void* X;
    char* Q;
    float* scale;
    int64_t M, K;       // of X
    int64_t rows, ld;   // of Q: rows, and bytes of one
    int64_t ns;         // scales of a block of 128 along a row of Q
    int64_t nk;         // blocks of 128 columns of X
};

// A workgroup quantises 128 columns of ROWS rows of X, sixteen lanes a row, eight values a lane, each read once and kept in
// registers between the maximum and the division.  Bound by memory: 8192 x 4096 in 19.5 us, 100 MB at 5.1 TB/s, as fast as a copy.
template <typename T, int BLOCK> __global__ __launch_bounds__(256) void quantize_rows_kernel(QuantArgs a) {
    constexpr int PASS = BLOCK == 128 ? 8 : 4, ROWS = 16 * PASS;
    __shared__ uint32_t most[4];
    const int tid = threadIdx.x, lane16 = tid & 15;
    const int64_t kb = blockIdx.x % a.nk, m0 = blockIdx.x / a.nk * ROWS, k = 128 * kb + 8 * lane16;
    float v[PASS][8];
    uint32_t top[PASS];
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
        const int64_t m = m0 + 16 * p + (tid >> 4);
        const u32x4 none = {0, 0, 0, 0};
        widen8<T>(m < a.M && k < a.K ? *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.X) + (m * a.K + k) * 2) : none, v[p]);
    }
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
        top[p] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top[p] = max(top[p], finite_magnitude(v[p][i]));
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) top[p] = max(top[p], (uint32_t)__shfl_xor((int)top[p], d));
    }
    if constexpr (BLOCK == 128) {
#pragma unroll
        for (int p = 1; p < PASS; ++p) top[0] = max(top[0], top[p]);
        top[0] = max(top[0], (uint32_t)__shfl_xor((int)top[0], 16));
        top[0] = max(top[0], (uint32_t)__shfl_xor((int)top[0], 32));
        if ((tid & 63) == 0) most[tid >> 6] = top[0];
        __syncthreads();
        top[0] = max(max(most[0], most[1]), max(most[2], most[3]));
#pragma unroll
        for (int p = 1; p < PASS; ++p) top[p] = top[0];
        if (tid == 0) a.scale[kb * a.ns + m0 / 128] = block_scale(top[0]);
    }
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
        const int64_t m = m0 + 16 * p + (tid >> 4);
        if (m >= a.M) break;
        const float s = block_scale(top[p]), inv = inverse_of_power(s);
        if (BLOCK == 1 && lane16 == 0) a.scale[kb * a.ns + m] = s;
        if (k < a.ld) *reinterpret_cast<uint2*>(a.Q + m * a.ld + k) = uint2{to_e4m3(v[p], inv), to_e4m3(v[p] + 4, inv)};
    }
}

// The transpose: a workgroup turns 128 rows x 128 columns of X into 128 bytes of 128 rows of Q, through LDS.  A thread
// takes 32 rows of two neighbouring columns, one LDS read for both.  8192 x 4096 in 25.6 us, 3.9 TB/s: 35 KB of LDS let four
// workgroups a CU overlap their reading, turning and writing, which is less than memory needs.
template <typename T, int BLOCK> __global__ __launch_bounds__(256) void quantize_columns_kernel(QuantArgs a) {
    constexpr int PITCH = 272;   // bytes of a row in LDS: 16-byte writes, and columns read by neighbouring lanes
    __shared__ __attribute__((aligned(16))) char tile[128 * PITCH];
    __shared__ uint2 most[256];
    const int tid = threadIdx.x;
    const int64_t kb = blockIdx.x % a.nk, mb = blockIdx.x / a.nk, m0 = 128 * mb, k0 = 128 * kb;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const int r = 16 * p + (tid >> 4), c = 8 * (tid & 15);
        const u32x4 none = {0, 0, 0, 0};
        const u32x4 w = m0 + r < a.M && k0 + c < a.K ? *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.X) + ((m0 + r) * a.K + k0 + c) * 2) : none;
        *reinterpret_cast<u32x4*>(tile + r * PITCH + 2 * c) = w;
    }
    __syncthreads();
    const int pair = tid & 63, quarter = tid >> 6;
    const char* from = tile + 32 * quarter * PITCH + 4 * pair;
    uint32_t w[32];
    uint2 top = {0, 0};
#pragma unroll
    for (int r = 0; r < 32; ++r) {
        w[r] = *reinterpret_cast<const uint32_t*>(from + r * PITCH);
        float lo, hi;
        unpack2<T>(w[r], lo, hi);
        top.x = max(top.x, finite_magnitude(lo));
        top.y = max(top.y, finite_magnitude(hi));
    }
    if constexpr (BLOCK == 128) {
        top.x = max(top.x, top.y);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) top.x = max(top.x, (uint32_t)__shfl_xor((int)top.x, d));
        top.y = top.x;
    }
    most[tid] = top;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        top.x = max(top.x, most[64 * q + pair].x);
        top.y = max(top.y, most[64 * q + pair].y);
    }
    const int64_t k = k0 + 2 * pair;
    const float s[2] = {block_scale(top.x), block_scale(top.y)};
    if (BLOCK == 128 ? tid == 0 : (quarter == 0 && k < a.K)) {
        a.scale[mb * a.ns + (BLOCK == 128 ? kb : k)] = s[0];
        if (BLOCK == 1) a.scale[mb * a.ns + k + 1] = s[1];
    }
    // the numbers go back through LDS (everybody has read the tile), so that rows of Q leave in whole lines
    constexpr int QP = 144;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const float inv = inverse_of_power(s[c]);
            u32x4 o;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float lo, hi;
                    unpack2<T>(w[16 * u + 4 * d + i], lo, hi);
                    v[i] = c ? hi : lo;
                }
                o[d] = to_e4m3(v, inv);
            }
            *reinterpret_cast<u32x4*>(tile + (2 * pair + c) * QP + 32 * quarter + 16 * u) = o;
        }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int r = 32 * p + (tid >> 3), at = 16 * (tid & 7);
        if (k0 + r < a.K && m0 + at < a.ld) *reinterpret_cast<u32x4*>(a.Q + (k0 + r) * a.ld + m0 + at) = *reinterpret_cast<const u32x4*>(tile + r * QP + at);
    }
}

// ---- launches ---------------------------------------------------------------------------------------------------
template <class G, class S> static hipError_t product(const Fp8Args& a, const Tile& t, int cus, hipStream_t st) {
    const int64_t items = most_row_blocks(a.R, a.E, G::BM) * ((a.N + G::BN - 1) / G::BN);
    hipLaunchKernelGGL((fp8_product_kernel<G, S>), dim3(persistent_grid(items, cus, t.per_cu)), dim3(64 * G::NW), group_table_bytes(a.E), st, a, t.cost);
    return hipGetLastError();
}
// Tiles, and their times for a block of 128 k, all set at one size (4096 x 4096 x 16384) with blocks of 128 of B's columns
static constexpr Tile kFp8[] = {{256, 256, 1, 1.68f, 2.0f, 4, 0.36f}, {128, 256, 1, 1.00f, 2.0f, 4, 0.39f}, {128, 128, 1, 0.58f, 2.0f, 2, 0.64f},
                                {64, 128, 1, 0.40f, 1.5f, 1, 1.0f},   {32, 128, 1, 0.33f, 1.5f, 1, 1.0f},   {64, 64, 2, 0.58f, 1.5f, 1, 1.0f}};
template <typename T, int MT> static hipError_t stream(const Fp8Args& a, hipStream_t st) {
    const int64_t items = most_row_blocks(a.R, a.E, 16 * MT) * ((a.N + 15) / 16);
    const dim3 grid((unsigned)((items + 7) / 8 * 8)), threads(512);
    const int table = a.offsets ? group_table_bytes(a.E) : 0;
    if (a.block == 1) hipLaunchKernelGGL((fp8_stream_kernel<T, MT, 1>), grid, threads, table, st, a);
    else hipLaunchKernelGGL((fp8_stream_kernel<T, MT, 128>), grid, threads, table, st, a);
    return hipGetLastError();
}
template <typename T, int BLOCK> static hipError_t tiles(const Fp8Args& a, int cus, hipStream_t st) {
    typedef Fp8Gemm<T, 256, 256, 2, 4, 2, BLOCK> G256;
    typedef Fp8Gemm<T, 128, 128, 4, 2, 4, BLOCK> G128;
    // (a ring of three: weights that come from memory are two steps away.  8192 uneven rows in 32 groups, 4096 x 2816: 181 us with
    // two stages, 153 with three)
    typedef Fp8Gemm<T, 128, 256, 2, 4, 3, BLOCK> W128;
    typedef Fp8Gemm<T, 64, 128, 2, 4, 5, BLOCK> G64;
    typedef Fp8Gemm<T, 32, 128, 1, 4, 6, BLOCK> G32;
    typedef Fp8Gemm<T, 64, 64, 2, 2, 4, BLOCK> S64;
    static_assert(G256::LDS_BYTES <= kLdsBesideGroups && G128::LDS_BYTES <= kLdsBesideGroups && G64::LDS_BYTES <= kLdsBesideGroups &&
                  G32::LDS_BYTES <= kLdsBesideGroups && S64::LDS_BYTES <= kLdsBesideGroups, "only W128 leaves less than the largest tables");
    static_assert(most_groups(S64::LDS_BYTES, kFp8[5].per_cu) >= kMaxGroups, "two workgroups a CU");
    const int i = pick_tile(kFp8, a.R, a.E, a.N, a.K, cus, a.E > kFp8Groups ? 1 : -1);
    switch (i) {
        case 0: return product<G256, G128>(a, kFp8[i], cus, st);
        case 1: return product<W128, G64>(a, kFp8[i], cus, st);
        case 2: return product<G128, G64>(a, kFp8[i], cus, st);
        case 3: return product<G64, G64>(a, kFp8[i], cus, st);
        case 4: return product<G32, G32>(a, kFp8[i], cus, st);
        default: return product<S64, S64>(a, kFp8[i], cus, st);
    }
}
template <typename T> static hipError_t product_any(const Fp8Args& a, int cus, hipStream_t st) {
    // Few rows: the streaming kernel, while its items are few enough to be under way together.  us, tiles -> this: one row of 4096 x
    // 11008 14.6 -> 13.8 (weights not in any cache), 11008 x 4096 29 -> 13, 2048 x 2048 8.2 -> 3.6, 8192 x 28672 46 -> 45; 32 rows of
    // 4096 x 4096 13.0 -> 8.6, of 4096 x 11008 13.4 -> 14.1.  512 rows in 64 groups 33 -> 84: each of many short items finds its group anew.
    const int64_t groups = a.R < a.E ? a.R : a.E, columns = (a.N + 15) / 16;
    if (a.R <= 16 * groups && most_row_blocks(a.R, a.E, 16) * columns <= (int64_t)8 * cus && (a.E == 1 || a.R <= 4 * groups)) return stream<T, 1>(a, st);
    if (a.E == 1 && a.R <= 32 && columns <= (int64_t)2 * cus) return stream<T, 2>(a, st);
    return a.block == 1 ? tiles<T, 1>(a, cus, st) : tiles<T, 128>(a, cus, st);
}
hipError_t launch_fp8_product(int dtype, const Fp8Args& a, int cus, hipStream_t st) {
    return dtype == 0 ? product_any<__bf16>(a, cus, st) : product_any<_Float16>(a, cus, st);
}

template <typename T> static hipError_t quantize(const QuantArgs& a, int block, bool transpose, hipStream_t st) {
    const int64_t rows = transpose || block == 128 ? 128 : 64;
    const dim3 grid((unsigned)(a.nk * ((a.M + rows - 1) / rows))), threads(256);
    if (transpose) {
        if (block == 1) hipLaunchKernelGGL((quantize_columns_kernel<T, 1>), grid, threads, 0, st, a);
        else hipLaunchKernelGGL((quantize_columns_kernel<T, 128>), grid, threads, 0, st, a);
    } else {
        if (block == 1) hipLaunchKernelGGL((quantize_rows_kernel<T, 1>), grid, threads, 0, st, a);
        else hipLaunchKernelGGL((quantize_rows_kernel<T, 128>), grid, threads, 0, st, a);
    }
    return hipGetLastError();
}
hipError_t launch_fp8_quantize(int dtype, const void* X, int64_t M, int64_t K, int block, bool transpose, void* Q, float* scale, hipStream_t st) {
    QuantArgs a{X, static_cast<char*>(Q), scale, M, K, 0, 0, 0, (K + 127) / 128};
    a.rows = transpose ? K : M;
    a.ld = ((transpose ? M : K) + 15) / 16 * 16;
    a.ns = (a.rows + block - 1) / block;
    return dtype == 0 ? quantize<__bf16>(a, block, transpose, st) : quantize<_Float16>(a, block, transpose, st);
}

}  // namespace ffuse
