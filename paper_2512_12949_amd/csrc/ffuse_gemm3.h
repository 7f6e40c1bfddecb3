// Block GEMMs whose two operands are laid out alike, beside DeepGemm and WideGemm (row operand contiguous along the
// contraction, weights across it): same accumulator layout, same epilogues.
//
//   RowGemm: both contiguous along the contraction (C = A B^T): a product's gradient of its input, dX = dY W^T.
//   ColGemm: both contiguous across it (C = A^T B): a product's gradient of its weights, dW = X^T dY.
#pragma once
#include "ffuse_gemm1.h"

namespace ffuse {

// One LDS-direct load, 16 bytes a lane, to LDS bytes [lds, lds + 1024).  In inline assembly, as in DeepGemm: the
// caller counts and waits for these loads itself.
__device__ __forceinline__ void lds_load16(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\tbuffer_load_dwordx4 %0, %2, 0 offen lds" :: "v"(voff), "s"(lds), "s"(r) : "memory", "m0");
}
template <int N> __device__ __forceinline__ void lds_loads_in_flight_at_most() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

// Both operands contiguous along the contraction.  A stage is 64 k of the BM + BN rows: rows of 128 bytes, a whole
// cache line, eight rows to a load instruction; 16-byte slot c of row r sits at position c ^ ((r >> 1) & 7), so that
// the sixteen rows a quarter of a wave reads together lie in sixteen different bank groups.  NS stages in a ring.
//
// A step multiplies one stage in four sub-steps of 16 k, the fragments of each read under the MFMAs of the one before.
// Before the last sub-step the loads of the next stage are waited for and the workgroup meets: everybody has read
// its last fragments of this stage, so the loads of the stage NS further on go into its place, under the last
// sub-step's MFMAs.  They have NS - 1 steps until they are waited for.
//
// Rows past the end of an operand repeat its last one (their products are never stored), so that no load is wholly out
// of range; chunks past the end of the contraction are out of range and read as zeros in both operands.
template <typename T, int BM, int BN, int WM, int WN, int NS>
struct RowGemm : FirstGemm<T, false, BM, BN, WM, WN> {
    typedef FirstGemm<T, false, BM, BN, WM, WN> Base;
    typedef typename Base::vec8 vec8;
    using Base::HT; using Base::MT; using Base::WHR; using Base::WMR;
    static constexpr int NW = WM * WN;
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "every wave issues the same number of loads");
    static constexpr int XI = BM / 8 / NW, BI = BN / 8 / NW, NLOAD = XI + BI;   // load instructions per wave and stage
    static constexpr int XB = BM * 128, STAGE = XB + BN * 128, LDS_BYTES = NS * STAGE;
    static_assert(NS >= 2 && (NS - 1) * NLOAD <= 63, "the vmcnt field holds 6 bits");
    static constexpr int NM = HT * MT, NR = HT + MT;
    static_assert(BM * BN * 2 <= LDS_BYTES, "the epilogue stages the tile");

    struct Ctx {
        __amdgpu_buffer_rsrc_t rx, rw;
        uint32_t xoff[XI], boff[BI];   // global byte offset of this lane's chunk at k = 0, per instruction
        int ck;                        // first k of this lane's chunk within a stage
        int K;
        uint32_t lds_a, lds_b;         // LDS offsets of this wave's first instruction
        uint32_t rdx[MT], rdw[HT];     // fragment reads, sub-step 0
    };
    // instruction q covers rows 8 q .. 8 q + 7; this wave's are q = wave, wave + NW, ...
    template <int N> static __device__ __forceinline__ void rows(uint32_t (&off)[N], int have, int64_t ld, int tid) {
        const int wave = tid >> 6, lane = tid & 63;
        const uint32_t chunk = (lane & 7u) ^ (uint32_t)(((wave & 1) << 2) | (lane >> 4));
#pragma unroll
        for (int j = 0; j < N; ++j) off[j] = (uint32_t)min(8 * (wave + NW * j) + (lane >> 3), have - 1) * (uint32_t)(2 * ld) + 16u * chunk;
    }
    // A: the block's first row, `have` rows of it exist; B likewise.  Both [rows][K].
    static __device__ __forceinline__ void aim(Ctx& c, const char* A, int have_a, const char* B, int have_b, int K, int tid) {
        have_a = min(have_a, BM); have_b = min(have_b, BN);
        c.rx = make_rsrc(A, (uint32_t)have_a * (uint32_t)(2 * K));
        c.rw = make_rsrc(B, (uint32_t)have_b * (uint32_t)(2 * K));
        c.K = K;
        rows<XI>(c.xoff, have_a, K, tid);
        rows<BI>(c.boff, have_b, K, tid);
    }
    static __device__ __forceinline__ void init_lds(Ctx& c, int tid) {
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
        const int wm = wave % WM, wn = wave / WM;
        const uint32_t x = lane & 31, h = lane >> 5;
        c.ck = 8 * ((lane & 7) ^ (((wave & 1) << 2) | (lane >> 4)));
        c.lds_a = (uint32_t)wave * 1024u;
        c.lds_b = XB + (uint32_t)wave * 1024u;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const uint32_t r = wm * WMR + 32 * mt + x;
            c.rdx[mt] = r * 128u + ((h ^ ((r >> 1) & 7u)) << 4);
        }
#pragma unroll
        for (int ht = 0; ht < HT; ++ht) {
            const uint32_t r = wn * WHR + 32 * ht + x;
            c.rdw[ht] = XB + r * 128u + ((h ^ ((r >> 1) & 7u)) << 4);
        }
    }
    static __device__ __forceinline__ void issue_one(const Ctx& c, uint32_t stage, int k, int i) {
        const bool ok = k + c.ck < c.K;
        if (i < XI) lds_load16(c.rx, ok ? c.xoff[i] + 2u * (uint32_t)k : kOob, stage + c.lds_a + (uint32_t)(i * NW) * 1024u);
        else lds_load16(c.rw, ok ? c.boff[i - XI] + 2u * (uint32_t)k : kOob, stage + c.lds_b + (uint32_t)((i - XI) * NW) * 1024u);
    }
    struct Frags {
        vec8 b[MT], a[HT];
    };
    static __device__ __forceinline__ void read_one(const char* stage, const Ctx& c, int ks, int i, Frags& f) {
        if (i == 0) f.b[0] = lds_read16<vec8>(stage, c.rdx[0] ^ (uint32_t)(ks << 5));
        else if (i <= HT) f.a[i - 1] = lds_read16<vec8>(stage, c.rdw[i - 1] ^ (uint32_t)(ks << 5));
        else f.b[i - HT] = lds_read16<vec8>(stage, c.rdx[i - HT] ^ (uint32_t)(ks << 5));
    }
    static __device__ __forceinline__ void run(char* smem, const Ctx& c, f32x16 (&acc)[HT][MT]) {
        f32x16 none[1][1];
        Base::zero(acc, none);
        const int KT = (c.K + 63) / 64;
        const uint32_t lds = (uint32_t)(uintptr_t)smem;
#pragma unroll
        for (int j = 0; j < NS; ++j)
            if (j < KT) {
#pragma unroll
                for (int i = 0; i < NLOAD; ++i) issue_one(c, lds + (uint32_t)(j * STAGE), 64 * j, i);
            }
        if (KT >= NS) lds_loads_in_flight_at_most<(NS - 1) * NLOAD>();
        else lds_loads_in_flight_at_most<0>();
        __syncthreads();
        Frags f[2];
#pragma unroll
        for (int i = 0; i < NR; ++i) read_one(smem, c, 0, i, f[0]);
        int slot = 0;
        for (int s = 0; s < KT; ++s) {
            const char* cur = smem + slot * STAGE;
            const uint32_t ld = lds + (uint32_t)(slot * STAGE);
            slot = slot == NS - 1 ? 0 : slot + 1;
            const char* nxt = smem + slot * STAGE;
#pragma unroll
            for (int ks = 0; ks < 3; ++ks)
#pragma unroll
                for (int i = 0; i < NM; ++i) {
                    acc[i / MT][i % MT] = Mma<T>::mma(f[ks & 1].a[i / MT], f[ks & 1].b[i % MT], acc[i / MT][i % MT]);
#pragma unroll
                    for (int e = (i * NR) / NM; e < ((i + 1) * NR) / NM; ++e) read_one(cur, c, ks + 1, e, f[(ks + 1) & 1]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            if (s + NS - 1 < KT) lds_loads_in_flight_at_most<(NS - 2) * NLOAD>();
            else lds_loads_in_flight_at_most<0>();
            __syncthreads();
            const bool more = s + NS < KT;
#pragma unroll
            for (int i = 0; i < NM; ++i) {
                acc[i / MT][i % MT] = Mma<T>::mma(f[1].a[i / MT], f[1].b[i % MT], acc[i / MT][i % MT]);
#pragma unroll
                for (int e = (i * NR) / NM; e < ((i + 1) * NR) / NM; ++e) read_one(nxt, c, 0, e, f[0]);
                if (more) {
#pragma unroll
                    for (int e = (i * NLOAD) / NM; e < ((i + 1) * NLOAD) / NM; ++e) issue_one(c, ld, 64 * (s + NS), e);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();   // LDS is the caller's
    }
};

// Both operands contiguous across the contraction.  A stage is 32 rows of the contraction x BM columns of the first
// and BN of the second operand, in their global orientation; both are transposed on the way out of LDS, as DeepGemm
// does with its weights (whose swizzle this is).  A ring of NS stages, a step of two sub-steps of 16 with one barrier
// between them, loads NS - 1 steps ahead.
//
// The base of the loads moves along with the steps, and so do the bytes that are left behind it: rows past the
// end read as zeros, offsets never pass 32 bits however long the contraction is.  A load instruction whose rows
// all lie past the end may complete ahead of older ones; where the last stage holds such rows, the steps that
// run while it is in flight wait for everything.
template <typename T, int BM, int BN, int WM, int WN, int NS>
struct ColGemm : FirstGemm<T, false, BM, BN, WM, WN> {
    typedef FirstGemm<T, false, BM, BN, WM, WN> Base;
    typedef typename Base::vec8 vec8;
    using Base::HT; using Base::MT; using Base::WHR; using Base::WMR;
    static constexpr int NW = WM * WN;
    static constexpr int XI = BM / 16 / NW, BI = BN / 16 / NW, NLOAD = XI + BI;   // 1 KB a load instruction
    static_assert(BM % (16 * NW) == 0 && BN % (16 * NW) == 0, "every wave issues the same number of loads");
    static constexpr int XB = BM * 64, STAGE = XB + BN * 64, LDS_BYTES = NS * STAGE;
    static_assert(NS >= 3 && (NS - 2) * NLOAD <= 63, "the vmcnt field holds 6 bits");
    static_assert(BM * BN * 2 <= LDS_BYTES, "the epilogue stages the tile");
    static constexpr int NM = HT * MT, NR = HT + MT;
    // XOR key of the 32-byte units of a row: the four rows of one transposing read in four different bank groups
    template <int COLS> static __device__ __forceinline__ uint32_t key(uint32_t k) {
        static_assert(COLS == 64 || COLS == 128 || COLS == 256, "rows of 4, 8 or 16 units of 32 bytes");
        return COLS == 64 ? (k & 2u) : ((k & 3u) << 1);
    }
    struct Ctx {
        const char *A, *B;             // the block's first column, row 0 of the contraction
        uint32_t lda, ldb;             // bytes of a row
        int rows;                      // of the contraction
        uint32_t xoff[XI], boff[BI];   // byte offset of this lane's chunk in a stage's rows (kOob: no such column)
        uint32_t lds_a, lds_b;
        uint32_t rdx[MT], rdw[HT];
    };
    template <int COLS, int N>
    static __device__ __forceinline__ void chunks(uint32_t (&off)[N], uint32_t ld, int have, int tid) {
        const int wave = tid >> 6, lane = tid & 63;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const uint32_t byte = (uint32_t)(wave * N + j) * 1024u + 16u * lane;
            const uint32_t k = byte / (2 * COLS), pp = (byte % (2 * COLS)) / 16u;
            const uint32_t p = (((pp >> 1) ^ key<COLS>(k)) << 1) | (pp & 1u);
            off[j] = (int)(8u * p) < have ? k * ld + 16u * p : kOob;
        }
    }
    // A: column `first of the block` of the first row, of which have_a columns exist; rows of lda / ldb elements
    static __device__ __forceinline__ void aim(Ctx& c, const char* A, int64_t lda, int have_a, const char* B, int64_t ldb, int have_b,
                                               int rows, int tid) {
        c.A = A; c.B = B;
        c.lda = (uint32_t)(2 * lda); c.ldb = (uint32_t)(2 * ldb);
        c.rows = rows;
        chunks<BM, XI>(c.xoff, c.lda, have_a, tid);
        chunks<BN, BI>(c.boff, c.ldb, have_b, tid);
    }
    static __device__ __forceinline__ void init_lds(Ctx& c, int tid) {
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
        const int wm = wave % WM, wn = wave / WM;
        c.lds_a = (uint32_t)(wave * XI) * 1024u;
        c.lds_b = XB + (uint32_t)(wave * BI) * 1024u;
        const uint32_t g = lane >> 4, jj = (lane >> 2) & 3u, q = lane & 3u;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const uint32_t u = (uint32_t)(wm * WMR + 32 * mt) / 16u + (g & 1u);
            c.rdx[mt] = (8u * (g >> 1) + jj) * (2 * BM) + ((u ^ key<BM>(jj)) * 32u) + 8u * q;
        }
#pragma unroll
        for (int ht = 0; ht < HT; ++ht) {
            const uint32_t u = (uint32_t)(wn * WHR + 32 * ht) / 16u + (g & 1u);
            c.rdw[ht] = XB + (8u * (g >> 1) + jj) * (2 * BN) + ((u ^ key<BN>(jj)) * 32u) + 8u * q;
        }
    }
    // the buffers of the stage whose first row is r (which exists)
    struct Src {
        __amdgpu_buffer_rsrc_t rx, rw;
    };
    static __device__ __forceinline__ Src source(const Ctx& c, int r) {
        const uint32_t n = (uint32_t)min(c.rows - r, 32);
        return {make_rsrc(c.A + (int64_t)r * c.lda, n * c.lda), make_rsrc(c.B + (int64_t)r * c.ldb, n * c.ldb)};
    }
    static __device__ __forceinline__ void issue_one(const Ctx& c, const Src& s, uint32_t stage, int i) {
        if (i < XI) lds_load16(s.rx, c.xoff[i], stage + c.lds_a + (uint32_t)i * 1024u);
        else lds_load16(s.rw, c.boff[i - XI], stage + c.lds_b + (uint32_t)(i - XI) * 1024u);
    }
    struct Frags {
        vec8 b[MT], a[HT];
    };
    template <int COLS> static __device__ __forceinline__ vec8 read_frag(const char* p) {
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 4 * 2 * COLS));
        typedef __attribute__((ext_vector_type(8))) short s16x8;
        const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(vec8, v);
    }
    static __device__ __forceinline__ void read_one(const char* stage, const Ctx& c, int ks, int i, Frags& f) {
        if (i == 0) f.b[0] = read_frag<BM>(stage + c.rdx[0] + ks * 16 * 2 * BM);
        else if (i <= HT) f.a[i - 1] = read_frag<BN>(stage + c.rdw[i - 1] + ks * 16 * 2 * BN);
        else f.b[i - HT] = read_frag<BM>(stage + c.rdx[i - HT] + ks * 16 * 2 * BM);
    }
    static __device__ __forceinline__ void run(char* smem, const Ctx& c, f32x16 (&acc)[HT][MT]) {
        f32x16 none[1][1];
        Base::zero(acc, none);
        const int KT = (c.rows + 31) / 32;
        if (KT == 0) return;
        const bool ragged = (c.rows & 31) != 0;
        const uint32_t lds = (uint32_t)(uintptr_t)smem;
#pragma unroll
        for (int j = 0; j < NS - 1; ++j)
            if (j < KT) {
                const Src s = source(c, 32 * j);
#pragma unroll
                for (int i = 0; i < NLOAD; ++i) issue_one(c, s, lds + (uint32_t)(j * STAGE), i);
            }
        // the steps that run while the last stage is in flight, or with fewer stages behind it, wait for everything
        if (KT >= NS || (KT == NS - 1 && !ragged)) lds_loads_in_flight_at_most<(NS - 2) * NLOAD>();
        else lds_loads_in_flight_at_most<0>();
        __syncthreads();
        Frags f[2];
#pragma unroll
        for (int i = 0; i < NR; ++i) read_one(smem, c, 0, i, f[0]);
        int slot = 0;
        for (int s = 0; s < KT; ++s) {
            const char* cur = smem + slot * STAGE;
            const uint32_t ld = lds + (uint32_t)((slot == 0 ? NS - 1 : slot - 1) * STAGE);
            slot = slot == NS - 1 ? 0 : slot + 1;
            const char* nxt = smem + slot * STAGE;
            const bool more = s + NS - 1 < KT;
            const Src src = source(c, more ? 32 * (s + NS - 1) : 0);
#pragma unroll
            for (int i = 0; i < NM; ++i) {
                acc[i / MT][i % MT] = Mma<T>::mma(f[0].a[i / MT], f[0].b[i % MT], acc[i / MT][i % MT]);
#pragma unroll
                for (int e = (i * NR) / NM; e < ((i + 1) * NR) / NM; ++e) read_one(cur, c, 1, e, f[1]);
                if (more) {
#pragma unroll
                    for (int e = (i * NLOAD) / NM; e < ((i + 1) * NLOAD) / NM; ++e) issue_one(c, src, ld, e);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // stages in flight behind the next one: s + 2 .. s + NS - 1, if they exist
            if (s + NS < KT || (s + NS == KT && !ragged)) lds_loads_in_flight_at_most<(NS - 2) * NLOAD>();
            else lds_loads_in_flight_at_most<0>();
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NM; ++i) {
                acc[i / MT][i % MT] = Mma<T>::mma(f[1].a[i / MT], f[1].b[i % MT], acc[i / MT][i % MT]);
#pragma unroll
                for (int e = (i * NR) / NM; e < ((i + 1) * NR) / NM; ++e) read_one(nxt, c, 0, e, f[0]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();   // LDS is the caller's
    }
};

}  // namespace ffuse
