// Block GEMM for products whose operands may lie either way in memory, beside DeepGemm and WideGemm (ffuse_gemm1.h, ffuse_gemm2.h):
// same accumulator layout.  C[BM][BN] = A B over a contraction of K, computed transposed (B's columns are the MFMA "A" operand).
//
//   ACOL = false: A[m][k], rows contiguous along the contraction       true: A[k][m]
//   BCOL = false: B[n][k]                                              true: B[k][n]   (GATED: two of them)
//
//   a product and its gradients:  Y = X W (false, true),  dX = dY W^T (false, false),  dW = X^T dY (true, true).
//
// A stage is 64 k of both operands, NS stages in a ring.  An operand contiguous along the contraction is kept as rows
// of 128 bytes, a whole cache line, eight rows to a load instruction; 16-byte slot c of row r sits at position
// c ^ ((r >> 1) & 7), so that the sixteen rows a quarter of a wave reads together lie in sixteen different bank groups.
// One contiguous across it is kept in its global orientation and transposed on the way out of LDS, with DeepGemm's swizzle.
//
// v_mfma_f32_16x16x32: on random operands, where the power limit sets the clock, its issue loop runs at 2.03 PFLOP/s and that of
// 32x32x16 at 1.75 (it reads and writes half as many accumulators per product).
//
// A step multiplies one stage, two halves of 32 k, 16 rows after 16 rows: the columns' fragments of a half stay in registers, a
// row block's are read two blocks ahead of their MFMAs.  Two row blocks before the step's end all its fragments are in
// registers: the next stage's loads are waited for and the workgroup meets; the loads of the stage NS further on go into this
// one's place under the MFMAs that are left, and so do the reads of the next step's first fragments.  The loads
// have NS - 1 steps until they are waited for.
//
// Past the end of the contraction both operands read as zeros.  Loads of stages past the last are issued all the same,
// out of range, so that every step has the same number in flight; rows past the end of an operand that is contiguous
// along the contraction repeat its last one (their products are not stored).
#pragma once
#include "ffuse_gemm1.h"

namespace ffuse {

// One LDS-direct load, 16 bytes a lane, to LDS bytes [lds, lds + 1024).  In inline assembly, as in DeepGemm: the
// caller counts and waits for these loads itself.
__device__ __forceinline__ void lds_load16(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\tbuffer_load_dwordx4 %0, %2, 0 offen lds" :: "v"(voff), "s"(lds), "s"(r) : "memory", "m0");
}
template <int N> __device__ __forceinline__ void lds_loads_in_flight_at_most() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

// 64 k of N rows or columns of an operand: its loads, dealt to NW waves, and its fragments
template <typename T, bool COL, int N, int NW> struct PairOperand;

template <typename T, int N, int NW> struct PairOperand<T, false, N, NW> {   // [n][k]
    static_assert(N % (8 * NW) == 0, "every wave issues the same number of loads");
    static constexpr int LOADS = N / 8 / NW, BYTES = N * 128;
    __amdgpu_buffer_rsrc_t r;
    uint32_t off[LOADS];   // of this lane's chunk at k = 0; instruction q of the operand covers rows 8 q .. 8 q + 7
    int ck, K;             // first k of the chunk within a stage; extent
    uint32_t dst, rd;
    // p: the first row, `have` rows of it exist, `ld` elements apart
    __device__ __forceinline__ void aim(const char* p, int64_t ld, int have, int k, int wave, int lane) {
        have = min(have, N);
        r = make_rsrc(p, (uint32_t)have * (uint32_t)(2 * ld));
        K = k;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) off[j] = (uint32_t)min(8 * (wave + NW * j) + (lane >> 3), have - 1) * (uint32_t)(2 * ld) + 2u * (uint32_t)ck;
    }
    __device__ __forceinline__ void init(uint32_t base, int first, int wave, int lane) {
        const uint32_t row = (uint32_t)first + (lane & 15), g = lane >> 4;
        ck = 8 * ((lane & 7) ^ (((wave & 1) << 2) | (lane >> 4)));
        dst = base + (uint32_t)wave * 1024u;
        rd = base + row * 128u + ((g ^ ((row >> 1) & 7u)) << 4);
    }
    __device__ __forceinline__ void load(uint32_t stage, int k, int j) const {
        lds_load16(r, k + ck < K ? off[j] + 2u * (uint32_t)k : kOob, stage + dst + (uint32_t)(j * NW) * 1024u);
    }
    // 16 rows x 32 k: rows 16 t on, half ks of the stage (the swizzle of a row repeats every 16)
    __device__ __forceinline__ typename Mma<T>::vec8 frag(const char* stage, int t, int ks) const {
        return lds_read16<typename Mma<T>::vec8>(stage, (rd ^ (uint32_t)(ks << 6)) + (uint32_t)t * 2048u);
    }
};

template <typename T, int N, int NW> struct PairOperand<T, true, N, NW> {   // [k][n]
    static_assert(N % (8 * NW) == 0 && (N == 64 || N == 128 || N == 256), "rows of 4, 8 or 16 units of 32 bytes");
    static constexpr int LOADS = N / 8 / NW, BYTES = N * 128, ROW = 2 * N;
    const char* p;
    uint32_t ld;           // bytes of a row
    uint32_t off[LOADS];   // of this lane's chunk within a stage's rows (kOob: no such column)
    int K;
    uint32_t dst, rd;
    // XOR key of the 32-byte units of a row.  Half a wave's transposing read touches one unit of the rows k, k + 1, k + 2, k + 3 and
    // of the four rows eight on: eight units in eight different bank groups (rows of 128 bytes alternate between two halves of
    // the banks by themselves).  Rows k and k + 4 have the same key.
    static __device__ __forceinline__ uint32_t key(uint32_t k) {
        return N == 64 ? ((k >> 1) & 1u) | ((k >> 2) & 2u) : (k & 3u) | ((k >> 1) & 4u);
    }
    // first: the first column, `have` columns exist; rows of `elems` elements
    __device__ __forceinline__ void aim(const char* first, int64_t elems, int have, int k, int wave, int lane) {
        p = first;
        ld = (uint32_t)(2 * elems);
        K = k;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const uint32_t byte = (uint32_t)(wave * LOADS + j) * 1024u + 16u * lane;
            const uint32_t row = byte / ROW, pp = (byte % ROW) / 16u;
            const uint32_t c = (((pp >> 1) ^ key(row)) << 1) | (pp & 1u);
            off[j] = (int)(8u * c) < have ? row * ld + 16u * c : kOob;
        }
    }
    __device__ __forceinline__ void init(uint32_t base, int first, int wave, int lane) {
        const uint32_t k = 8u * (lane >> 4) + ((lane >> 2) & 3u);
        dst = base + (uint32_t)(wave * LOADS) * 1024u;
        rd = base + k * ROW + (((uint32_t)first / 16u) ^ key(k)) * 32u + 8u * (lane & 3u);
    }
    // (the base moves along with the stages, and with it the bytes that are left: rows past the end are out of range, and
    // offsets never pass 32 bits however long the contraction is)
    __device__ __forceinline__ void load(uint32_t stage, int k, int j) const {
        const int left = min(K - k, 64);
        lds_load16(make_rsrc(p + (int64_t)k * ld, left > 0 ? (uint32_t)left * ld : 0u), off[j], stage + dst + (uint32_t)j * 1024u);
    }
    // 16 columns x 32 k: columns 16 t on, half ks.  (Units t on: `first` leaves the bits of t zero, so a XOR, like the key.)
    __device__ __forceinline__ typename Mma<T>::vec8 frag(const char* stage, int t, int ks) const {
        const char* a = stage + (rd ^ (uint32_t)(t << 5)) + ks * 32 * ROW;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(a));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(a + 4 * ROW));
        typedef __attribute__((ext_vector_type(8))) short s16x8;
        const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(typename Mma<T>::vec8, v);
    }
};

// D[16][16] += A[16][32] B[16][32]^T: lane l holds row l % 16 and k = 8 (l / 16) .. + 7 of either operand, and of D column l % 16,
// rows 4 (l / 16) + r.
template <typename T> __device__ __forceinline__ f32x4 mma16(typename Mma<T>::vec8 a, typename Mma<T>::vec8 b, f32x4 c);
template <> __device__ __forceinline__ f32x4 mma16<__bf16>(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
template <> __device__ __forceinline__ f32x4 mma16<_Float16>(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// The activations of the products by expert: as everywhere, but ReLU leaves NaN as it is, where the chains of one expert make it
// zero.  v_maximum3_f32, one instruction as there.
template <int ACT> __device__ __forceinline__ float activate_keep_nan(float x) {
    return ACT == ACT_RELU ? __builtin_elementwise_maximum(x, 0.0f) : activate<ACT>(x);
}

// A tile of accumulators of 16 x 16 products (computed transposed: a lane has four neighbouring columns of a row) on its way out:
// 16 rows of a wave's COLS columns at a time through LDS of the wave's own, so that a row's part is stored in one piece.
// Every wave issues MT * STORES stores, those of rows and columns that do not exist out of range.
template <typename T, int COLS, int MT> struct TileStore {
    static constexpr int HT = COLS / 16, ROW = 2 * COLS, LPR = ROW / 16, RPI = 64 / LPR, SLOTS = ROW / 8, LDS_BYTES = 16 * ROW, STORES = 16 / RPI;
    static_assert(COLS == 32 || COLS == 64, "rows of 64 or 128 bytes");
    // value(ht, mt, r): column 16 ht + 4 (lane / 16) + r of row 16 mt + lane % 16 of the wave's block, whose first row is row0 and first
    // column col0 of a tile of have_m x have_n at C
    template <class Value>
    static __device__ __forceinline__ void store(char* mine, char* C, uint32_t ldc, int row0, int col0, int rows, int have_m, int have_n, Value&& value) {
        int lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
        asm volatile("" : "+v"(lane));   // (otherwise the addresses below are computed before the main loop and kept through it)
        const uint32_t x = lane & 15, g = lane >> 4, rin = lane / LPR, ch = lane % LPR;
        constexpr int SHIFT = ROW == 128 ? 1 : 2;   // log2 of the rows in 256 bytes: those lie in different banks by themselves
        const uint32_t key = (x >> SHIFT) & (SLOTS - 1);
        const int col = col0 + 8 * (int)ch;
        const __amdgpu_buffer_rsrc_t rc = make_rsrc(C, (uint32_t)min(have_m, rows) * 2u * ldc);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
            for (int ht = 0; ht < HT; ++ht) {
                float v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = value(ht, mt, r);
                *reinterpret_cast<uint2*>(mine + x * ROW + (((4 * ht + g) ^ key) << 3)) = uint2{pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3])};
            }
#pragma unroll
            for (int i = 0; i < STORES; ++i) {
                const uint32_t row = (uint32_t)(i * RPI) + rin, k = (row >> SHIFT) & (SLOTS - 1);
                u32x4 v = *reinterpret_cast<const u32x4*>(mine + row * ROW + ((ch ^ (k >> 1)) << 4));
                if (k & 1u) v = u32x4{v[2], v[3], v[0], v[1]};
                const int m = row0 + 16 * mt + (int)row;
                __builtin_amdgcn_raw_buffer_store_b128(v, rc, m < have_m && col < have_n ? ((uint32_t)m * ldc + (uint32_t)col) * 2u : kOob, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

template <typename T, bool ACOL, bool BCOL, bool GATED, int BM_, int BN_, int WM, int WN, int NS> struct PairGemm {
    typedef typename Mma<T>::vec8 vec8;
    static constexpr int BM = BM_, BN = BN_;
    static constexpr int NW = WM * WN, G = GATED ? 2 : 1;
    static constexpr int WMR = BM / WM, WNR = BN / WN, MT = WMR / 16, HT = WNR / 16;   // a wave's rows, columns and 16 x 16 tiles
    static_assert(WMR % 32 == 0 && WNR % 16 == 0, "16 x 16 tiles, an even number of row blocks");
    typedef PairOperand<T, ACOL, BM, NW> OpA;
    typedef PairOperand<T, BCOL, BN, NW> OpB;
    static constexpr int NLOAD = OpA::LOADS + G * OpB::LOADS, STAGE = OpA::BYTES + G * OpB::BYTES;
    // (a wave's columns leave 32 at a time where the ring leaves no room for 64; 8 KB are the group tables')
    static constexpr int ECOL = WNR == 64 && NS * STAGE + NW * 2048 > 152 * 1024 ? 32 : WNR;
    typedef TileStore<T, ECOL, MT> Store;
    static constexpr int EPI = NS * STAGE, LDS_BYTES = EPI + NW * Store::LDS_BYTES, STORES = WNR / ECOL * MT * Store::STORES;
    static_assert(NS >= 2 && (NS - 1) * NLOAD + STORES <= 63, "the vmcnt field holds 6 bits");
    static constexpr int NB = 2 * MT, NM = G * HT;   // row blocks of a step, MFMAs of each

    struct Ctx {
        OpA a;
        OpB b[G];
        int K;
    };
    static __device__ __forceinline__ void init(Ctx& c, int wave, int lane) {
        const int wm = wave % WM, wn = wave / WM;
        c.a.init(0u, wm * WMR, wave, lane);
#pragma unroll
        for (int g = 0; g < G; ++g) c.b[g].init(OpA::BYTES + (uint32_t)g * OpB::BYTES, wn * WNR, wave, lane);
    }
    static __device__ __forceinline__ void issue_one(const Ctx& c, uint32_t stage, int k, int i) {
        if (i < OpA::LOADS) c.a.load(stage, k, i);
        else c.b[(i - OpA::LOADS) / OpB::LOADS].load(stage, k, (i - OpA::LOADS) % OpB::LOADS);
    }
    // the loads of an item's first NS stages
    static __device__ __forceinline__ void fill(char* smem, const Ctx& c) {
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int i = 0; i < NLOAD; ++i) issue_one(c, (uint32_t)(uintptr_t)smem + (uint32_t)(j * STAGE), 64 * j, i);
    }
    // filled: the item's first stages were issued before the epilogue of the item before, whose STORES stores are younger
    static __device__ __forceinline__ void run(char* smem, const Ctx& c, f32x4 (&acc)[G][HT][MT], bool filled) {
#pragma unroll
        for (int i = 0; i < NM * MT; ++i) acc[i / MT / HT][i / MT % HT][i % MT] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int KT = (c.K + 63) / 64;
        const uint32_t lds = (uint32_t)(uintptr_t)smem;
        if (filled) lds_loads_in_flight_at_most<(NS - 1) * NLOAD + STORES>();
        else lds_loads_in_flight_at_most<(NS - 1) * NLOAD>();
        __syncthreads();
        // of either half the columns' fragments; of the last four row blocks read theirs.  Block i of a step is half i / MT, rows i % MT.
        vec8 a[2][G][HT], b[4];
        b[0] = c.a.frag(smem, 0, 0);
#pragma unroll
        for (int j = 0; j < NM; ++j) a[0][j % G][j / G] = c.b[j % G].frag(smem, j / G, 0);
        b[1] = c.a.frag(smem, 1, 0);
        int slot = 0;
        for (int s = 0; s < KT; ++s) {
            const char* cur = smem + slot * STAGE;
            const uint32_t ld = lds + (uint32_t)(slot * STAGE);
            slot = slot == NS - 1 ? 0 : slot + 1;
            const char* nxt = smem + slot * STAGE;
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                if (i == NB - 2) {
                    lds_loads_in_flight_at_most<(NS - 2) * NLOAD>();
                    __syncthreads();
                }
#pragma unroll
                for (int j = 0; j < NM; ++j) {
                    const int g = j % G, ht = j / G;
                    acc[g][ht][i % MT] = mma16<T>(a[i / MT][g][ht], b[i & 3], acc[g][ht][i % MT]);
                    if (j == 0) {
                        const int n = i + 2;   // the row block to read
                        b[n & 3] = n < NB ? c.a.frag(cur, n % MT, n / MT) : c.a.frag(nxt, n - NB, 0);
                    }
                    if (i < MT) {              // the second half's columns, spread over the first half
#pragma unroll
                        for (int e = (i * NM + j) / MT; e < (i * NM + j + 1) / MT; ++e) a[1][e % G][e / G] = c.b[e % G].frag(cur, e / G, 1);
                    }
                    if (i >= NB - 2) {
                        const int p = (i - NB + 2) * NM + j;   // of the last 2 NM products
                        if (p < NM) a[0][p % G][p / G] = c.b[p % G].frag(nxt, p / G, 0);
#pragma unroll
                        for (int e = p * NLOAD / (2 * NM); e < (p + 1) * NLOAD / (2 * NM); ++e) issue_one(c, ld, 64 * (s + NS), e);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        __syncthreads();   // the stages are the next item's
    }

    // C: the tile's first row and column, rows of ldc elements, of which have_m rows and have_n columns exist (a multiple of 8)
    template <int ACT>
    static __device__ __forceinline__ void store(char* smem, const f32x4 (&acc)[G][HT][MT], char* C, uint32_t ldc, int have_m, int have_n, int wave) {
#pragma unroll
        for (int e = 0; e < WNR / ECOL; ++e)
            Store::store(smem + EPI + wave * Store::LDS_BYTES, C, ldc, wave % WM * WMR, wave / WM * WNR + e * ECOL, BM, have_m, have_n, [&](int h, int mt, int r) {
                const int ht = e * (ECOL / 16) + h;
                const float v = activate_keep_nan<ACT>(acc[0][ht][mt][r]);
                return GATED ? v * acc[G - 1][ht][mt][r] : v;
            });
    }
    static __device__ __forceinline__ void store_rt(char* smem, int act, const f32x4 (&acc)[G][HT][MT], char* C, uint32_t ldc, int have_m, int have_n, int wave) {
        switch (act) {
            case ACT_RELU: store<ACT_RELU>(smem, acc, C, ldc, have_m, have_n, wave); break;
            case ACT_GELU_TANH: store<ACT_GELU_TANH>(smem, acc, C, ldc, have_m, have_n, wave); break;
            case ACT_SILU: store<ACT_SILU>(smem, acc, C, ldc, have_m, have_n, wave); break;
            default: store<ACT_IDENTITY>(smem, acc, C, ldc, have_m, have_n, wave); break;
        }
    }
};

}  // namespace ffuse
