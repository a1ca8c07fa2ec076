// 4-bit floating point: the stored form of a quantised matrix, and the groups of its rows.
//
// An element is e2m1 (0 .5 1 1.5 2 3 4 6 and a sign), two to a byte, the even one in the low nibble.  Blocks of 32 (e8m0) or 16
// (e4m3) elements of a row share a scale byte.  Scales lie in tiles of 512 bytes, 128 rows x 4 blocks, as the
// tensor core wants them in its memory: byte (r % 32) * 16 + (r / 32) * 4 + b.  The rows of group g start at
// row 0 of tile offsets[g] / 128 + g: that is never before the end of group g - 1's tiles, and takes no table of the groups.
#pragma once

#include "bnn_common.cuh"

namespace bnn {
namespace f4 {

constexpr int kMaxGroups = 1024;
constexpr int kMaxK = 1 << 24;
// SMs that fixed thresholds and the plan of the router go by: the size of a workspace may not change with the current device.
constexpr int kSms = 148;

__host__ __device__ __forceinline__ int block_of(int format) { return format == BNN_F4_E8M0_32 ? 32 : 16; }
// bytes of a row of codes
__host__ __device__ __forceinline__ int code_bytes(int K) { return ((K + 31) >> 5) * 16; }
// scale tiles along K
__host__ __device__ __forceinline__ int scale_tiles(int format, int K) { return ceil_div(K, 4 * block_of(format)); }
// row tiles of a matrix of `rows` rows in `groups` groups
__host__ __device__ __forceinline__ int row_tiles(int rows, int groups) { return rows / 128 + groups; }

// Group of a row: the last g < G with offsets[g] <= row.  A whole warp asks; two dependent loads for up to 1024 groups.
// False where the row is in no group (behind the last one, or offsets that make no sense).
__device__ __forceinline__ bool find_group(const int32_t* __restrict__ offsets, int G, int row, int lane, int* group, int* first) {
    int coarse = lane * 32, at = 0;
    const unsigned c = __ballot_sync(0xFFFFFFFFu, coarse < G && __ldg(offsets + coarse) <= row);
    if (c == 0) return false;
    coarse = (31 - __clz(c)) * 32;
    const int mine = coarse + lane;
    const int off = mine < G ? __ldg(offsets + mine) : 0x7FFFFFFF;
    const unsigned f = __ballot_sync(0xFFFFFFFFu, mine < G && off <= row);
    if (f == 0) return false;
    const int l = 31 - __clz(f);
    at = __shfl_sync(0xFFFFFFFFu, off, l);
    *group = coarse + l;
    *first = at;
    return at >= 0 && row < __ldg(offsets + coarse + l + 1);
}

}  // namespace f4

struct F4QuantArgs {
    const void* X;             // [src_rows][ldx] of dtype
    int dtype, src_rows, ldx;
    const int32_t* source;     // [rows] or nullptr: row r is X[source[r]]
    const int32_t* offsets;    // [groups + 1] or nullptr
    int groups, rows, K, format;
    float factor;              // power of two that the values are multiplied by first
    uint8_t* codes;
    int ldc;
    uint8_t* scales;
};
int launch_f4_quantize(const F4QuantArgs& a, cudaStream_t st);

struct F4DequantArgs {
    const uint8_t* codes;
    int ldc;
    const uint8_t* scales;
    const int32_t* offsets;
    int groups, rows, K, format;
    float factor;
    void* Y;
    int dtype, ldy;
};
int launch_f4_dequantize(const F4DequantArgs& a, cudaStream_t st);

struct F4GemmArgs {
    const uint8_t* a;          // codes [M][lda]
    int lda;
    const uint8_t* a_scales;
    const int32_t* offsets;    // [groups + 1] or nullptr (one group of M rows)
    int groups;
    const uint8_t* w;          // codes [groups * N][ldw]
    int ldw;
    const uint8_t* w_scales;
    int M, N, K, format;
    float factor;              // power of two that the sums are multiplied by
    const float* scale;        // [groups][N] or nullptr
    const float* shift;
    int act, sign_mode;
    void* Y;                   // [M][ldy] of dtype, or nullptr
    int dtype, ldy;
    uint32_t* out_bits;        // [M][ldob], or nullptr
    int ldob;
};
int launch_f4_gemm(const F4GemmArgs& a, cudaStream_t st);
int f4_gemm_form(int M, int N, int K, int groups, int sms, bnn_f4_form* form);

struct RouteArgs {
    const void* logits;
    int dtype, T, E, ld, k, mode;
    int32_t* index;
    float* weight;
    int32_t* offsets;
    int32_t* slot;
    int32_t* source;
    void* workspace;
};
size_t route_workspace_bytes(int T, int E);
int launch_route(const RouteArgs& a, cudaStream_t st);

struct CombineArgs {
    const void* Z;
    int dtype, ldz, rows;
    const int32_t* slot;
    const float* weight;
    int T, k, N;
    void* Y;
    int y_dtype, ldy;
};
int launch_combine(const CombineArgs& a, cudaStream_t st);

}  // namespace bnn
