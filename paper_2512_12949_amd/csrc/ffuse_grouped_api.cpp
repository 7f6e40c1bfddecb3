// C-ABI layer of the products grouped by expert and of the 8-bit products: argument validation and launches.  See
// include/ffuse.h for the contract of every entry point.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/ffuse.h"
#include "ffuse_launch.h"

namespace {

constexpr int64_t kMaxExperts = 1024;      // group boundaries are kept in LDS
constexpr int64_t kMaxWidth = 1 << 20;     // 256 rows of an operand stay below 2 GiB: they are addressed by 32-bit offsets

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool width_ok(int64_t n) { return n >= 8 && n % 8 == 0 && n <= kMaxWidth; }

// R rows in E groups, one K x N matrix each; `elem` bytes an element.  Work items are numbered by 32-bit integers.
bool groups_ok(int64_t R, int64_t E, int64_t K, int64_t N, int elem) {
    if (E < 1 || E > kMaxExperts || R < 0 || R >= ((int64_t)1 << 31) - 512) return false;
    if (!width_ok(K) || !width_ok(N)) return false;
    if ((K + 128) * N * elem >= (int64_t)1 << 31) return false;
    return (R / 16 + E) * (std::max(K, N) / 32 + 1) < (int64_t)1 << 31;
}

// what a forward product and the input's gradient need alike: A and C are empty when there are no rows
int check_grouped(int dtype, const void* A, const void* W, const void* W3, const void* offsets, int64_t R, int64_t E, int64_t K, int64_t N,
                  const void* C) {
    if (!W || !offsets || (R != 0 && (!A || !C))) return FFUSE_ERR_NULL;
    if (dtype != FFUSE_DT_BF16 && dtype != FFUSE_DT_F16) return FFUSE_ERR_ACT;
    if (!groups_ok(R, E, K, N, 2)) return FFUSE_ERR_SHAPE;
    if (!aligned(A, 16) || !aligned(W, 16) || !aligned(W3, 16) || !aligned(C, 16) || !aligned(offsets, 4)) return FFUSE_ERR_ALIGN;
    return FFUSE_OK;
}

int status(hipError_t e) { return e == hipSuccess ? FFUSE_OK : FFUSE_ERR_LAUNCH; }

ffuse::GroupedArgs grouped_args(const void* A, const void* W, const void* W3, const void* offsets, void* C, int64_t R, int64_t E, int64_t K,
                                int64_t N, int act) {
    return {A, W, W3, static_cast<const int32_t*>(offsets), C, (int)R, (int)E, (int)K, (int)N, act};
}

int fp8_product(int dtype, const void* A, const float* sa, const void* B, const float* sb, int b_block, const int32_t* offsets, int64_t R,
                int64_t E, int64_t K, int64_t N, void* Y, void* stream) {
    if (!B || !sb || (R != 0 && (!A || !sa || !Y))) return FFUSE_ERR_NULL;
    if (dtype != FFUSE_DT_BF16 && dtype != FFUSE_DT_F16) return FFUSE_ERR_ACT;
    if (b_block != 1 && b_block != 128) return FFUSE_ERR_SHAPE;
    if (K % 16 || !groups_ok(R, E, K, N, 1)) return FFUSE_ERR_SHAPE;
    if (!aligned(A, 16) || !aligned(B, 16) || !aligned(Y, 16) || !aligned(sa, 4) || !aligned(sb, 4) || !aligned(offsets, 4)) return FFUSE_ERR_ALIGN;
    int cus = 0;
    const int rc = ffuse::device_ready(&cus);
    if (rc != FFUSE_OK || R == 0) return rc;
    const ffuse::Fp8Args a{A, sa, B, sb, offsets, Y, (int)R, (int)E, (int)K, (int)N, b_block};
    return status(ffuse::launch_fp8_product(dtype, a, cus, static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

int ffuse_grouped_gemm(int dtype, const void* X, const void* W, const void* W3, const int32_t* offsets, int act, int64_t R, int64_t E, int64_t K,
                       int64_t N, void* Y, void* stream) {
    int rc = check_grouped(dtype, X, W, W3, offsets, R, E, K, N, Y);
    if (rc != FFUSE_OK) return rc;
    if (act < FFUSE_ACT_IDENTITY || act > FFUSE_ACT_SILU) return FFUSE_ERR_ACT;
    int cus = 0;
    rc = ffuse::device_ready(&cus);
    if (rc != FFUSE_OK || R == 0) return rc;
    return status(ffuse::launch_grouped_forward(dtype, grouped_args(X, W, W3, offsets, Y, R, E, K, N, act), cus, static_cast<hipStream_t>(stream)));
}

int ffuse_grouped_gemm_dx(int dtype, const void* dY, const void* W, const int32_t* offsets, int64_t R, int64_t E, int64_t K, int64_t N, void* dX,
                          void* stream) {
    int rc = check_grouped(dtype, dY, W, nullptr, offsets, R, E, K, N, dX);
    if (rc != FFUSE_OK) return rc;
    int cus = 0;
    rc = ffuse::device_ready(&cus);
    if (rc != FFUSE_OK || R == 0) return rc;
    return status(ffuse::launch_grouped_input(dtype, grouped_args(dY, W, nullptr, offsets, dX, R, E, K, N, 0), cus, static_cast<hipStream_t>(stream)));
}

int ffuse_grouped_gemm_dw(int dtype, const void* X, const void* dY, const int32_t* offsets, int64_t R, int64_t E, int64_t K, int64_t N, void* dW,
                          void* stream) {
    if (!offsets || !dW || (R != 0 && (!X || !dY))) return FFUSE_ERR_NULL;
    if (dtype != FFUSE_DT_BF16 && dtype != FFUSE_DT_F16) return FFUSE_ERR_ACT;
    // (a launch holds fewer than 2^32 threads: 2^23 blocks of 128 x 128)
    if (!groups_ok(R, E, K, N, 2) || E * ((K + 127) / 128) * ((N + 127) / 128) >= (int64_t)1 << 23) return FFUSE_ERR_SHAPE;
    if (!aligned(X, 16) || !aligned(dY, 16) || !aligned(dW, 16) || !aligned(offsets, 4)) return FFUSE_ERR_ALIGN;
    int cus = 0;
    const int rc = ffuse::device_ready(&cus);
    if (rc != FFUSE_OK) return rc;
    return status(ffuse::launch_grouped_weights(dtype, grouped_args(X, dY, nullptr, offsets, dW, R, E, K, N, 0), cus, static_cast<hipStream_t>(stream)));
}

size_t ffuse_grouped_workspace_bytes(int dtype, int64_t R, int64_t N1) {
    if ((dtype != FFUSE_DT_BF16 && dtype != FFUSE_DT_F16) || R < 0 || R >= (int64_t)1 << 31 || !width_ok(N1)) return 0;
    return ((size_t)R * (size_t)N1 * 2 + 255) / 256 * 256;
}

int ffuse_grouped_ffn(int dtype, const void* X, const void* W1, const void* W3, const void* W2, const int32_t* offsets, int act, int64_t R, int64_t E,
                      int64_t K, int64_t N1, int64_t N2, void* Y, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_grouped(dtype, X, W1, W3, offsets, R, E, K, N1, Y);
    if (rc != FFUSE_OK) return rc;
    rc = check_grouped(dtype, X, W2, nullptr, offsets, R, E, N1, N2, Y);
    if (rc != FFUSE_OK) return rc;
    if (act < FFUSE_ACT_IDENTITY || act > FFUSE_ACT_SILU) return FFUSE_ERR_ACT;
    int cus = 0;
    rc = ffuse::device_ready(&cus);
    if (rc != FFUSE_OK || R == 0) return rc;
    if (!workspace || workspace_bytes < (size_t)R * (size_t)N1 * 2) return FFUSE_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return FFUSE_ERR_ALIGN;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    // H in 16 bits, as in the chains of one expert: it is an operand of the second product's matrix instructions, which take no more.
    // (The chain's error against 64 bits is 1.4 times that of one rounding of the result: 0.0023 and 0.0017 of its size in bf16.)
    const ffuse::WorkspaceWrite write(workspace, workspace_bytes, st);
    rc = status(ffuse::launch_grouped_forward(dtype, grouped_args(X, W1, W3, offsets, workspace, R, E, K, N1, act), cus, st));
    if (rc != FFUSE_OK) return rc;
    return status(ffuse::launch_grouped_forward(dtype, grouped_args(workspace, W2, nullptr, offsets, Y, R, E, N1, N2, FFUSE_ACT_IDENTITY), cus, st));
}

int ffuse_fp8_quantize(int dtype, const void* X, int64_t M, int64_t K, int block_rows, int transpose, void* Q, float* scale, void* stream) {
    if (M != 0 && (!X || !Q || !scale)) return FFUSE_ERR_NULL;
    if (dtype != FFUSE_DT_BF16 && dtype != FFUSE_DT_F16) return FFUSE_ERR_ACT;
    if (block_rows != 1 && block_rows != 128) return FFUSE_ERR_SHAPE;
    // (a launch holds fewer than 2^32 threads: a workgroup quantises 64 rows of 128 columns at least)
    if (M < 0 || !width_ok(K) || M >= (int64_t)1 << 31 || (M / 64 + 1) * (K / 128 + 1) >= (int64_t)1 << 23) return FFUSE_ERR_SHAPE;
    if (!aligned(X, 16) || !aligned(Q, 16) || !aligned(scale, 4)) return FFUSE_ERR_ALIGN;
    int cus = 0;
    const int rc = ffuse::device_ready(&cus);
    if (rc != FFUSE_OK || M == 0) return rc;
    return status(ffuse::launch_fp8_quantize(dtype, X, M, K, block_rows, transpose != 0, Q, scale, static_cast<hipStream_t>(stream)));
}

int ffuse_gemm_fp8(int dtype, const void* A, const float* sa, const void* B, const float* sb, int b_block, int64_t M, int64_t K, int64_t N, void* Y,
                   void* stream) {
    return fp8_product(dtype, A, sa, B, sb, b_block, nullptr, M, 1, K, N, Y, stream);
}

int ffuse_grouped_gemm_fp8(int dtype, const void* A, const float* sa, const void* B, const float* sb, int b_block, const int32_t* offsets, int64_t R,
                           int64_t E, int64_t K, int64_t N, void* Y, void* stream) {
    if (!offsets) return FFUSE_ERR_NULL;
    return fp8_product(dtype, A, sa, B, sb, b_block, offsets, R, E, K, N, Y, stream);
}

}  // extern "C"
