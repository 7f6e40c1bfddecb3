// Matrix products grouped by expert: rows sorted by expert, a weight matrix for each.
//
//   forward : Y[r] = act(X[r] W[e]) [.* X[r] W3[e]]     X [R][K], W [E][K][N]
//   input   : dX[r] = dY[r] W[e]^T                       dY [R][N]
//   weights : dW[e] = X_e^T dY_e                         zeros for a group without rows
//
// The boundaries of the groups are on the device (ffuse_groups.h), so the host knows neither how many row blocks
// there are nor whose they are: forward and input run persistent workgroups, which each lay the row blocks of all
// groups end to end and take their share; a weight gradient's blocks are known beforehand.
#include "ffuse_gemm2.h"
#include "ffuse_gemm3.h"
#include "ffuse_groups.h"
#include "ffuse_launch.h"

namespace ffuse {

// ---- forward ----------------------------------------------------------------------------------------------------
template <typename T, typename G, int BM, int BH, int THREADS>
__global__ __launch_bounds__(THREADS) void grouped_forward_kernel(GroupedArgs a) {
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    extern __shared__ __attribute__((aligned(16))) char table[];
    const int tid = threadIdx.x, xcd = blockIdx.x & 7, step = gridDim.x >> 3;
    Groups groups;
    scan_groups(groups, table, a.offsets, a.E, a.R, BM, tid);
    f32x16 acc[G::HT][G::MT], acc3[G::G == 2 ? G::HT : 1][G::G == 2 ? G::MT : 1];
    typename G::Ctx c;
    G::init_lds(c, tid);
    const int ncol = (a.N + BH - 1) / BH;
    const int64_t wbytes = 2 * (int64_t)a.K * a.N;
    GroupItem it;
    for (int idx = blockIdx.x >> 3; group_item(groups, BM, ncol, xcd, idx, it); idx += step) {
        const int rows = min(it.rows, BM);
        const char* X = static_cast<const char*>(a.A) + it.row0 * a.K * 2;
        const char* W = static_cast<const char*>(a.W) + it.e * wbytes;
        const char* W3 = G::G == 2 ? static_cast<const char*>(a.W3) + it.e * wbytes : nullptr;
        G::init_a(c, X, (uint32_t)rows * (uint32_t)(2 * a.K), 0u, 0u, (uint32_t)a.K, a.K, tid);
        G::init_b(c, W, W3, (uint32_t)wbytes, (uint32_t)a.N, (uint32_t)a.N, (uint32_t)(it.col * BH), tid);
        G::run(smem, c, 0, a.K, acc, acc3, tid);
        char* Y = static_cast<char*>(a.C) + it.row0 * a.N * 2;
        if constexpr (BM == 256) G::store_tile_slabs_rt(smem, a.act, acc, acc3, Y, a.N, 0, it.col * BH, rows, a.N, __builtin_amdgcn_readfirstlane(tid >> 6));
        else G::store_tile_lds_rt(smem, a.act, acc, acc3, Y, a.N, 0, it.col * BH, rows, a.N, tid);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
}

// ---- gradient of the input --------------------------------------------------------------------------------------
template <typename T, int BM, int BN, int WM, int WN, int NS>
__global__ __launch_bounds__(64 * WM * WN) void grouped_input_kernel(GroupedArgs a) {
    typedef RowGemm<T, BM, BN, WM, WN, NS> G;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    extern __shared__ __attribute__((aligned(16))) char table[];
    const int tid = threadIdx.x, xcd = blockIdx.x & 7, step = gridDim.x >> 3;
    Groups groups;
    scan_groups(groups, table, a.offsets, a.E, a.R, BM, tid);
    f32x16 acc[G::HT][G::MT], none[1][1];
    typename G::Ctx c;
    G::init_lds(c, tid);
    const int ncol = (a.K + BN - 1) / BN;
    GroupItem it;
    for (int idx = blockIdx.x >> 3; group_item(groups, BM, ncol, xcd, idx, it); idx += step) {
        const int col0 = it.col * BN;
        G::aim(c, static_cast<const char*>(a.A) + it.row0 * a.N * 2, it.rows,
               static_cast<const char*>(a.W) + ((int64_t)it.e * a.K + col0) * a.N * 2, a.K - col0, a.N, tid);
        G::run(smem, c, acc);
        char* dX = static_cast<char*>(a.C) + it.row0 * a.K * 2;
        G::template store_tile_lds<ACT_IDENTITY>(smem, acc, none, dX, a.K, 0, col0, min(it.rows, BM), a.K, tid);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
}

// ---- gradient of the weights ------------------------------------------------------------------------------------
// One block of one group's gradient a workgroup, in order of the groups: the hardware hands them out as CUs come
// free, which evens out groups of different lengths.
template <typename T, int BM, int BN, int WM, int WN, int NS>
__global__ __launch_bounds__(64 * WM * WN) void grouped_weights_kernel(GroupedArgs a) {
    typedef ColGemm<T, BM, BN, WM, WN, NS> G;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    const int tid = threadIdx.x;
    const int mb = (a.K + BM - 1) / BM, nb = (a.N + BN - 1) / BN;
    const int e = (int)(blockIdx.x / (uint32_t)(mb * nb)), b = (int)(blockIdx.x % (uint32_t)(mb * nb));
    // (any boundaries are taken: the rows read are inside the tensor, and nothing but dW[e] is written)
    const int first = min(max(a.offsets[e], 0), a.R), last = min(max(a.offsets[e + 1], 0), a.R);
    const int rows = max(last - first, 0);
    const int band = b / (kGroupBand * nb), in = b - band * kGroupBand * nb, h = min(kGroupBand, mb - band * kGroupBand);
    const int m0 = (band * kGroupBand + in % h) * BM, n0 = in / h * BN;
    f32x16 acc[G::HT][G::MT], none[1][1];
    typename G::Ctx c;
    G::init_lds(c, tid);
    G::aim(c, static_cast<const char*>(a.A) + ((int64_t)first * a.K + m0) * 2, a.K, a.K - m0,
           static_cast<const char*>(a.W) + ((int64_t)first * a.N + n0) * 2, a.N, a.N - n0, rows, tid);
    G::run(smem, c, acc);
    char* dW = static_cast<char*>(a.C) + (int64_t)e * a.K * a.N * 2;
    G::template store_tile_lds<ACT_IDENTITY>(smem, acc, none, dW, a.N, m0, n0, a.K, a.N, tid);
}

// ---- launches ---------------------------------------------------------------------------------------------------
template <typename T, typename G, int BM, int BH, int THREADS> static hipError_t forward(const GroupedArgs& a, int cus, int per_cu, hipStream_t st) {
    const int grid = persistent_grid(most_row_blocks(a.R, a.E, BM) * ((a.N + BH - 1) / BH), cus, per_cu);
    hipLaunchKernelGGL((grouped_forward_kernel<T, G, BM, BH, THREADS>), dim3(grid), dim3(THREADS), group_table_bytes(a.E), st, a);
    return hipGetLastError();
}
template <typename T> static hipError_t forward_any(const GroupedArgs& a, int cus, hipStream_t st) {
    if (a.W3) return forward<T, WideGemm<T, true, 128, 128, 4, 2, 4>, 128, 128, 512>(a, cus, 1, st);
    return forward<T, WideGemm<T, false, 128, 256, 2, 4, 4>, 128, 256, 512>(a, cus, 1, st);
}
hipError_t launch_grouped_forward(int dtype, const GroupedArgs& a, int cus, hipStream_t st) {
    return dtype == 0 ? forward_any<__bf16>(a, cus, st) : forward_any<_Float16>(a, cus, st);
}

template <typename T, int BM, int BN, int WM, int WN, int NS> static hipError_t input(const GroupedArgs& a, int cus, int per_cu, hipStream_t st) {
    const int grid = persistent_grid(most_row_blocks(a.R, a.E, BM) * ((a.K + BN - 1) / BN), cus, per_cu);
    hipLaunchKernelGGL((grouped_input_kernel<T, BM, BN, WM, WN, NS>), dim3(grid), dim3(64 * WM * WN), group_table_bytes(a.E), st, a);
    return hipGetLastError();
}
template <typename T> static hipError_t input_any(const GroupedArgs& a, int cus, hipStream_t st) {
    return input<T, 128, 128, 2, 2, 4>(a, cus, 1, st);
}
hipError_t launch_grouped_input(int dtype, const GroupedArgs& a, int cus, hipStream_t st) {
    return dtype == 0 ? input_any<__bf16>(a, cus, st) : input_any<_Float16>(a, cus, st);
}

template <typename T, int BM, int BN, int WM, int WN, int NS> static hipError_t weights(const GroupedArgs& a, hipStream_t st) {
    const int64_t grid = (int64_t)a.E * ((a.K + BM - 1) / BM) * ((a.N + BN - 1) / BN);
    hipLaunchKernelGGL((grouped_weights_kernel<T, BM, BN, WM, WN, NS>), dim3((unsigned)grid), dim3(64 * WM * WN), 0, st, a);
    return hipGetLastError();
}
template <typename T> static hipError_t weights_any(const GroupedArgs& a, hipStream_t st) {
    return weights<T, 128, 128, 2, 2, 4>(a, st);
}
hipError_t launch_grouped_weights(int dtype, const GroupedArgs& a, hipStream_t st) {
    return dtype == 0 ? weights_any<__bf16>(a, st) : weights_any<_Float16>(a, st);
}

}  // namespace ffuse
