// Quantisation to 4-bit floating point and back.
//
// A block of n elements (32 or 16) shares a scale s:  q = round(x / s) to the nearest e2m1 number, ties to the even code, what is
// beyond 6 becomes 6;  e8m0: s = 2^(floor(log2 max|x|) - 2), so that the largest element lands in [4, 8);  e4m3: s = max|x| / 6
// rounded to the nearest e4m3 number (at most 448; a block whose s rounds to 0 becomes zeros).  Every decision is that of the
// exact quotient: the division by a power of two is exact, and a quotient rounded to 24 bits by a scale of four bits lies on
// a border between two codes only if the exact one does (a border times s has seven bits; the next fp32 number is
// further off than half a step of the quotient).  Blocks with a NaN or an infinity get the scale NaN.
//
// Bound by memory: 8 elements a lane, 256 a warp and turn; the block's maximum is an integer maximum of magnitudes over two or
// four lanes (NaNs are the largest).  A lane writes 4 bytes of codes, the first lane of a block the scale's byte.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "f4.cuh"

namespace bnn {
namespace {

constexpr int WARPS = 8;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }

// Eight consecutive elements from p (n of them exist, n <= 0: none).
template <bool VEC>
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8]) {
    if (VEC && n >= 8) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? __ldg(p + i) : 0.0f;
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T* p, int n, float (&v)[8]) {
    if (VEC && n >= 8) {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(p));
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            T h[2];
            memcpy(h, &w[i], 4);
            v[2 * i] = to_f32(h[0]);
            v[2 * i + 1] = to_f32(h[1]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? to_f32(p[i]) : 0.0f;
    }
}

// Eight numbers -> eight codes, the first in the lowest nibble: to the nearest, ties to even, beyond 6 becomes 6.
__device__ __forceinline__ uint32_t to_codes(const float (&v)[8]) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}

// fp32 >= 0 -> e4m3 byte, to the nearest, ties to even, at most 448; and back.
__device__ __forceinline__ uint32_t to_e4m3(float x) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(x));
    return r & 0xFFu;
}
__device__ __forceinline__ float from_e4m3(uint32_t b) {      // sign bit clear
    const uint32_t e = b >> 3, m = b & 7u;
    if (b == 0x7Fu) return __uint_as_float(0x7FC00000u);
    return e ? __uint_as_float(((e + 120u) << 23) | (m << 20)) : (float)m * 0x1p-9f;
}
__device__ __forceinline__ float from_e8m0(uint32_t b) {
    return b == 0xFFu ? __uint_as_float(0x7FC00000u) : b ? __uint_as_float(b << 23) : 0x1p-127f;
}

__device__ __forceinline__ size_t scale_place(int tile, int kt, int katom, int row) {
    return ((size_t)tile * kt + katom) * 512 + (size_t)((row & 31) * 16 + ((row & 127) >> 5) * 4);
}

// Tile and row inside it of row r (warp-uniform); false: the row belongs to no group.
__device__ __forceinline__ bool locate(const int32_t* offsets, int groups, int row, int lane, int* tile, int* local) {
    int g = 0, first = 0;
    if (offsets && !f4::find_group(offsets, groups, row, lane, &g, &first)) return false;
    *local = row - first;
    *tile = first / 128 + g + *local / 128;
    return true;
}

// Largest magnitude of eight elements as the bits of an fp32 number (NaNs are above all others).
__device__ __forceinline__ uint32_t magnitude(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return m;
}
// The same from eight 16-bit elements as they were loaded, two at a time.
__device__ __forceinline__ uint32_t magnitude2(const uint4& w) {
    const uint32_t keep = 0x7FFF7FFFu;
    const uint32_t m = __vmaxu2(__vmaxu2(w.x & keep, w.y & keep), __vmaxu2(w.z & keep, w.w & keep));
    return max(m & 0xFFFFu, m >> 16);
}
__device__ __forceinline__ uint32_t widen_magnitude(uint32_t m, __nv_bfloat16) { return m << 16; }
__device__ __forceinline__ uint32_t widen_magnitude(uint32_t m, __half) { return __float_as_uint(__half2float(__ushort_as_half((unsigned short)m))); }

// One block's share of a lane: eight elements and the block's largest magnitude -> codes, and the scale's byte.
template <bool MX>
__device__ __forceinline__ uint32_t to_block(float (&v)[8], uint32_t most, uint32_t* scale) {
    const bool finite = most < 0x7F800000u;
    uint32_t byte, codes;
    if (MX) {
        byte = max(most >> 23, 2u) - 2u;
        const float inverse = __uint_as_float((254u - byte) << 23);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= inverse;
        codes = to_codes(v);
    } else {
        byte = to_e4m3(__fdiv_rn(__uint_as_float(most), 6.0f));
        const float s = from_e4m3(byte), inverse = __frcp_rn(s);
        // The quotient to the nearest from the rounded reciprocal (Markstein, IBM J. Res. Dev. 34, 1990): the remainder
        // is exact in a fused multiply-add, and one correction rounds as a division does.  (It makes +0 of -0.)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float q = v[i] * inverse;
            v[i] = copysignf(byte ? __fmaf_rn(__fmaf_rn(-q, s, v[i]), inverse, q) : 0.0f, v[i]);
        }
        codes = to_codes(v);
    }
    *scale = finite ? byte : MX ? 0xFFu : 0x7Fu;
    return finite ? codes : 0u;
}

template <bool MX>
__device__ __forceinline__ uint32_t block_max(uint32_t m) {
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
    if (MX) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
    return m;
}

// A warp: UNROLL segments of 256 elements of a row.
template <typename T, bool MX, bool VEC, int UNROLL>
__global__ void __launch_bounds__(WARPS * 32) quantize_kernel(const __grid_constant__ F4QuantArgs g, int turns, long long items) {
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const long long item = (long long)blockIdx.x * WARPS + (threadIdx.x >> 5);
    if (item >= items) return;
    const int row = (int)(item / turns), first = (int)(item - (long long)row * turns) * UNROLL * 256;
    const int src = g.source ? __ldg(g.source + row) : row;
    const T* x = static_cast<const T*>(g.X) + (long long)src * g.ldx + first + lane * 8;
    const bool there = !g.source || (src >= 0 && src < g.src_rows);
    constexpr int LANES = MX ? 4 : 2;                     // lanes of a block
    const int k0 = first + lane * 8, kt = f4::scale_tiles(g.format, g.K);
    int tile, local;
    // a lane's blocks are 256 / (8 LANES) apart, as many as fill 256 / (32 LANES) tiles
    constexpr int TILES = 256 / (32 * LANES);
    const int block = k0 / (8 * LANES);
    if (VEC && there && first + UNROLL * 256 <= g.K) {
        // all of it exists: no test on the way
        if constexpr (sizeof(T) == 2) {
            uint4 raw[UNROLL];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) raw[u] = __ldg(reinterpret_cast<const uint4*>(x + u * 256));
            if (!locate(g.offsets, g.groups, row, lane, &tile, &local)) return;
            uint8_t* codes = g.codes + (size_t)row * g.ldc + (k0 >> 1);
            uint8_t* scales = g.scales + scale_place(tile, kt, block >> 2, local) + (block & 3);
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                float v[8];
                const uint32_t w[4] = {raw[u].x, raw[u].y, raw[u].z, raw[u].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    T h[2];
                    memcpy(h, &w[i], 4);
                    v[2 * i] = to_f32(h[0]);
                    v[2 * i + 1] = to_f32(h[1]);
                }
                uint32_t most;
                if (g.factor == 1.0f) {
                    most = widen_magnitude(block_max<MX>(magnitude2(raw[u])), T());
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] *= g.factor;
                    most = block_max<MX>(magnitude(v));
                }
                uint32_t byte;
                *reinterpret_cast<uint32_t*>(codes + u * 128) = to_block<MX>(v, most, &byte);
                if (lane % LANES == 0) scales[u * TILES * 512] = (uint8_t)byte;
            }
        } else {
            float v[UNROLL][8];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) load8<true>(x + u * 256, 8, v[u]);
            if (!locate(g.offsets, g.groups, row, lane, &tile, &local)) return;
            uint8_t* codes = g.codes + (size_t)row * g.ldc + (k0 >> 1);
            uint8_t* scales = g.scales + scale_place(tile, kt, block >> 2, local) + (block & 3);
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[u][i] *= g.factor;
                uint32_t byte;
                const uint32_t most = block_max<MX>(magnitude(v[u]));
                *reinterpret_cast<uint32_t*>(codes + u * 128) = to_block<MX>(v[u], most, &byte);
                if (lane % LANES == 0) scales[u * TILES * 512] = (uint8_t)byte;
            }
        }
        return;
    }
    if (!locate(g.offsets, g.groups, row, lane, &tile, &local)) return;
    const int bytes = f4::code_bytes(g.K);
#pragma unroll 1
    for (int u = 0; u < UNROLL; ++u) {
        const int k = k0 + u * 256;
        float v[8];
        load8<VEC>(x + u * 256, there ? g.K - k : 0, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= g.factor;
        uint32_t byte;
        const uint32_t codes = to_block<MX>(v, block_max<MX>(magnitude(v)), &byte);
        if (k >> 1 < bytes) *reinterpret_cast<uint32_t*>(g.codes + (size_t)row * g.ldc + (k >> 1)) = codes;
        const int b = block + u * TILES * 4;
        if (lane % LANES == 0 && b >> 2 < kt) g.scales[scale_place(tile, kt, b >> 2, local) + (b & 3)] = k < g.K ? (uint8_t)byte : (uint8_t)0;
    }
}

// Two codes -> two numbers.
__device__ __forceinline__ float2 from_codes(uint32_t pair) {
    uint32_t h;
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}" : "=r"(h) : "r"(pair));
    __half2 p;
    memcpy(&p, &h, 4);
    return __half22float2(p);
}

__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__half* p, float v) { *p = __float2half_rn(v); }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

template <bool VEC>
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
    if (VEC && n >= 8) {
        reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = v[i];
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* p, int n, const float (&v)[8]) {
    if (VEC && n >= 8) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            T h[2];
            put(&h[0], v[2 * i]);
            put(&h[1], v[2 * i + 1]);
            memcpy(&w[i], h, 4);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) put(p + i, v[i]);
    }
}

template <typename T, bool MX, bool VEC, int UNROLL>
__global__ void __launch_bounds__(WARPS * 32) dequantize_kernel(const __grid_constant__ F4DequantArgs g, int turns, long long items) {
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const long long item = (long long)blockIdx.x * WARPS + (threadIdx.x >> 5);
    if (item >= items) return;
    const int row = (int)(item / turns), first = (int)(item % turns) * UNROLL * 256;
    const int kt = f4::scale_tiles(g.format, g.K);
    uint32_t codes[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const int k = first + u * 256 + lane * 8;
        codes[u] = k < g.K ? __ldg(reinterpret_cast<const uint32_t*>(g.codes + (size_t)row * g.ldc + (k >> 1))) : 0u;
    }
    int tile, local;
    if (!locate(g.offsets, g.groups, row, lane, &tile, &local)) return;
    const int k0 = first + lane * 8, block = k0 / (MX ? 32 : 16);
    constexpr int TILES = MX ? 2 : 4;          // of scales in a segment
    T* y = static_cast<T*>(g.Y) + (long long)row * g.ldy + k0;
    const uint8_t* scales = g.scales + scale_place(tile, kt, block >> 2, local) + (block & 3);
    uint32_t byte[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) byte[u] = k0 + u * 256 < g.K ? __ldg(scales + u * TILES * 512) : 0u;
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const int n = g.K - k0 - u * 256;
        if (n <= 0) continue;
        const float s = MX ? from_e8m0(byte[u]) : from_e4m3(byte[u] & 0x7Fu);
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = from_codes(codes[u] >> (8 * i));
            v[2 * i] = p.x * s;
            v[2 * i + 1] = p.y * s;
        }
        if (g.factor != 1.0f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= g.factor;
        }
        store8<VEC>(y + u * 256, n, v);
    }
}

template <typename A>
using Kernel = void (*)(A, int, long long);

template <typename T, bool VEC, int U>
Kernel<F4QuantArgs> quantizer(int format) {
    return format == BNN_F4_E8M0_32 ? quantize_kernel<T, true, VEC, U> : quantize_kernel<T, false, VEC, U>;
}
template <typename T, bool VEC, int U>
Kernel<F4DequantArgs> dequantizer(int format) {
    return format == BNN_F4_E8M0_32 ? dequantize_kernel<T, true, VEC, U> : dequantize_kernel<T, false, VEC, U>;
}
template <typename T>
Kernel<F4QuantArgs> pick(const F4QuantArgs& a, bool vec, bool many) {
    if (many) return vec ? quantizer<T, true, 4>(a.format) : quantizer<T, false, 4>(a.format);
    return vec ? quantizer<T, true, 1>(a.format) : quantizer<T, false, 1>(a.format);
}
template <typename T>
Kernel<F4DequantArgs> pick(const F4DequantArgs& a, bool vec, bool many) {
    if (many) return vec ? dequantizer<T, true, 4>(a.format) : dequantizer<T, false, 4>(a.format);
    return vec ? dequantizer<T, true, 1>(a.format) : dequantizer<T, false, 1>(a.format);
}

template <typename A>
int launch(const A& a, const void* real, int dtype, int ld, cudaStream_t st) {
    const int size = dtype == BNN_DTYPE_F32 ? 4 : 2;
    const bool vec = aligned16(real) && ((long long)ld * size) % 16 == 0;
    const int segments = ceil_div(a.K, 256);
    // Four segments a warp where there is enough for every SM's warps, so that a lane has four loads in flight.
    const bool many = (long long)a.rows * segments >= 4LL * 148 * 64 && segments >= 4;
    const int turns = ceil_div(segments, many ? 4 : 1);
    const long long items = (long long)a.rows * turns, grid = (items + WARPS - 1) / WARPS;
    if (grid > 0x7FFFFFFF) return BNN_ERR_SHAPE;
    Kernel<A> kern = dtype == BNN_DTYPE_F32 ? pick<float>(a, vec, many)
                   : dtype == BNN_DTYPE_F16 ? pick<__half>(a, vec, many) : pick<__nv_bfloat16>(a, vec, many);
    if (launch_pdl(kern, dim3((unsigned)grid), dim3(WARPS * 32), 0, st, a, turns, items) != cudaSuccess) return BNN_ERR_CUDA;
    return launch_status();
}

}  // namespace

int launch_f4_quantize(const F4QuantArgs& a, cudaStream_t st) { return launch(a, a.X, a.dtype, a.ldx, st); }
int launch_f4_dequantize(const F4DequantArgs& a, cudaStream_t st) { return launch(a, a.Y, a.dtype, a.ldy, st); }

}  // namespace bnn
