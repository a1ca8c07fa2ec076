// Quantisation to 4-bit floating point and back.
//
// A block of n elements (32 or 16) shares a scale s:  q = round(x / s) to the nearest e2m1 number, ties to the even code, what is
// beyond 6 becomes 6;  e8m0: s = 2^(floor(log2 max|x|) - 2), so that the largest element lands in [4, 8);  e4m3: s = max|x| / 6
// rounded to the nearest e4m3 number (at most 448; a block whose s rounds to 0 becomes zeros).  Every decision is that of the
// exact quotient: the division by a power of two is exact, and a quotient rounded to 24 bits by a scale of four bits lies on
// a border between two codes only if the exact one does (a border times s has seven bits; the next fp32 number is
// further off than half a step of the quotient).  Blocks with a NaN or an infinity get the scale NaN.
//
// Bound by memory where rows are read once: 16384 x 4096 bf16 take 25 us (172 MB, 6.9 TB/s), back 27 us (6.3 TB/s).  Gathered rows come mostly
// from L2 and are bound by instructions (16384 from 4096 rows 24 us).  The block's
// maximum is an integer maximum of magnitudes over its lanes (NaNs are the largest), two 16-bit ones at a time.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

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
__device__ __forceinline__ uint32_t to_codes(const float* v) {
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

// Sixteen consecutive elements from p (32-byte aligned) by 32-byte loads.
__device__ __forceinline__ void ldg32(const void* p, uint32_t (&w)[8]) {
    asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
}
template <typename T> struct Sixteen {
    uint32_t w[8];
    __device__ __forceinline__ void load(const T* p) { ldg32(p, w); }
    __device__ __forceinline__ void values(float (&v)[16]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            T h[2];
            memcpy(h, &w[i], 4);
            v[2 * i] = to_f32(h[0]);
            v[2 * i + 1] = to_f32(h[1]);
        }
    }
    // the largest magnitude as the bits of an fp32 number, two elements at a time
    __device__ __forceinline__ uint32_t magnitude() const {
        uint32_t m = w[0] & 0x7FFF7FFFu;
#pragma unroll
        for (int i = 1; i < 8; ++i) m = __vmaxu2(m, w[i] & 0x7FFF7FFFu);
        m = max(m & 0xFFFFu, m >> 16);
        return std::is_same<T, __half>::value ? __float_as_uint(__half2float(__ushort_as_half((unsigned short)m))) : m << 16;
    }
};
template <> struct Sixteen<float> {
    uint32_t w[16];
    __device__ __forceinline__ void load(const float* p) {
        ldg32(p, reinterpret_cast<uint32_t(&)[8]>(w[0]));
        ldg32(p + 8, reinterpret_cast<uint32_t(&)[8]>(w[8]));
    }
    __device__ __forceinline__ void values(float (&v)[16]) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(w[i]);
    }
    __device__ __forceinline__ uint32_t magnitude() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max(m, w[i] & 0x7FFFFFFFu);
        return m;
    }
};

// Largest magnitude of N elements as the bits of an fp32 number (NaNs are above all others).
template <int N>
__device__ __forceinline__ uint32_t magnitude(const float (&v)[N]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return m;
}

// One block's share of a lane: N elements and the block's largest magnitude -> codes, eight to a word, and the scale's byte.
template <bool MX, int N>
__device__ __forceinline__ void to_block(float (&v)[N], uint32_t most, uint32_t (&codes)[N / 8], uint32_t* scale) {
    const bool finite = most < 0x7F800000u;
    uint32_t byte;
    if (MX) {
        byte = max(most >> 23, 2u) - 2u;
        const float inverse = __uint_as_float((254u - byte) << 23);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] *= inverse;
    } else {
        byte = to_e4m3(__fdiv_rn(__uint_as_float(most), 6.0f));
        const float s = from_e4m3(byte), inverse = __frcp_rn(s);
        // The quotient to the nearest from the rounded reciprocal (Markstein, IBM J. Res. Dev. 34, 1990): the remainder
        // is exact in a fused multiply-add, and one correction rounds as a division does.  (It makes +0 of -0.)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float q = v[i] * inverse;
            v[i] = copysignf(byte ? __fmaf_rn(__fmaf_rn(-q, s, v[i]), inverse, q) : 0.0f, v[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
        codes[i] = to_codes(&v[8 * i]);
        if (!finite) codes[i] = 0u;
    }
    *scale = finite ? byte : MX ? 0xFFu : 0x7Fu;
}

// A warp: SEGMENT elements of a row; the warps of a block: rows one behind the other.  WIDE (32-byte aligned rows): a lane has 16
// consecutive elements twice where all of the segment exists, which is half of an e8m0 block or a whole e4m3 block; else 8 and
// tests on the way.
constexpr int SEGMENT = 1024;
template <typename T, bool MX, bool VEC, bool WIDE>
__global__ void __launch_bounds__(WARPS * 32) quantize_kernel(const __grid_constant__ F4QuantArgs g, int segment) {
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int row = blockIdx.x * WARPS + (threadIdx.x >> 5), first = blockIdx.y * segment;
    if (row >= g.rows) return;
    const int src = g.source ? __ldg(g.source + row) : row;
    const T* x = static_cast<const T*>(g.X) + (long long)src * g.ldx + first;
    const bool there = !g.source || (src >= 0 && src < g.src_rows);
    const int kt = f4::scale_tiles(g.format, g.K);
    constexpr int BLOCK = MX ? 32 : 16;
    int tile, local;
    if (WIDE && there && first + SEGMENT <= g.K) {       // (segment == SEGMENT)
        Sixteen<T> raw[2];
        raw[0].load(x + lane * 16);
        raw[1].load(x + 512 + lane * 16);
        if (!locate(g.offsets, g.groups, row, lane, &tile, &local)) return;
        const int k0 = first + lane * 16, block = k0 / BLOCK;
        uint8_t* codes = g.codes + (size_t)row * g.ldc + (k0 >> 1);
        uint8_t* scales = g.scales + scale_place(tile, kt, block >> 2, local) + (block & 3);
        const bool writer = !MX || !(lane & 1);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float v[16];
            raw[u].values(v);
            uint32_t most;
            if (g.factor == 1.0f) {
                most = raw[u].magnitude();
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] *= g.factor;
                most = magnitude(v);
            }
            if (MX) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
            uint32_t c[2], byte;
            to_block<MX>(v, most, c, &byte);
            *reinterpret_cast<uint2*>(codes + u * 256) = make_uint2(c[0], c[1]);
            if (writer) scales[u * (128 / BLOCK) * 512] = (uint8_t)byte;
        }
        return;
    }
    if (!locate(g.offsets, g.groups, row, lane, &tile, &local)) return;
    const int bytes = f4::code_bytes(g.K);
#pragma unroll 1
    for (int s = 0; s < segment; s += 256) {
        const int k = first + s + lane * 8, block = k / BLOCK;
        float v[8];
        load8<VEC>(x + s + lane * 8, there ? g.K - k : 0, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= g.factor;
        uint32_t most = magnitude(v);
        most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
        if (MX) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
        uint32_t c[1], byte;
        to_block<MX>(v, most, c, &byte);
        if (k >> 1 < bytes) *reinterpret_cast<uint32_t*>(g.codes + (size_t)row * g.ldc + (k >> 1)) = c[0];
        if (k % BLOCK == 0 && block >> 2 < kt) g.scales[scale_place(tile, kt, block >> 2, local) + (block & 3)] = k < g.K ? (uint8_t)byte : (uint8_t)0;
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

// Four codes (16 bits) -> four bf16, two to a word.  The bytes of the eight magnitudes come from tables of eight bytes by byte permutation,
// whose selector is the code itself; a selector's bit 3 (the sign) makes it replicate the byte's top bit, which tells 0x80 from 0xFF.
__device__ __forceinline__ void to_bf16(uint32_t codes, uint32_t* first, uint32_t* second) {
    const uint32_t mag = codes & 0x7777u;
    const uint32_t lo = __byte_perm(0xC0800000u, 0xC0804000u, mag);     // 0 .5 1 1.5 | 2 3 4 6: 0000 3F00 3F80 3FC0 4000 4040 4080 40C0
    uint32_t hi = __byte_perm(0x3F3F3F00u, 0x40404040u, mag);
    uint32_t sign;
    asm("prmt.b32 %0, %1, %1, %2;" : "=r"(sign) : "r"(0x80808080u), "r"(codes));
    hi |= (sign << 1) & 0x80808080u;
    *first = __byte_perm(lo, hi, 0x5140);
    *second = __byte_perm(lo, hi, 0x7362);
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    __nv_bfloat162 x, y;
    memcpy(&x, &a, 4);
    memcpy(&y, &b, 4);
    x = __hmul2(x, y);
    memcpy(&a, &x, 4);
    return a;
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
__global__ void __launch_bounds__(WARPS * 32) dequantize_kernel(const __grid_constant__ F4DequantArgs g) {
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int row = blockIdx.x * WARPS + (threadIdx.x >> 5), first = blockIdx.y * UNROLL * 256;
    if (row >= g.rows) return;
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
        if constexpr (VEC && sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value) {
            if (n >= 8) {
                // a code times a scale has at most six bits: exact in bf16, whose exponents are those of fp32
                uint32_t w[4];
                to_bf16(codes[u] & 0xFFFFu, &w[0], &w[1]);
                to_bf16(codes[u] >> 16, &w[2], &w[3]);
                // (the factor first: that product neither overflows nor underflows, so that all is rounded once)
                if (g.factor != 1.0f) {
                    const uint32_t f2 = (__float_as_uint(g.factor) >> 16) * 0x10001u;
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = mul_bf16x2(w[i], f2);
                }
                const uint32_t s2 = (__float_as_uint(s) >> 16) * 0x10001u;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = mul_bf16x2(w[i], s2);
                *reinterpret_cast<uint4*>(y + u * 256) = make_uint4(w[0], w[1], w[2], w[3]);
                continue;
            }
        }
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = from_codes(codes[u] >> (8 * i));
            v[2 * i] = p.x * g.factor * s;
            v[2 * i + 1] = p.y * g.factor * s;
        }
        store8<VEC>(y + u * 256, n, v);
    }
}

template <typename T, bool VEC, bool WIDE>
void (*quantizer(int format))(F4QuantArgs, int) {
    return format == BNN_F4_E8M0_32 ? quantize_kernel<T, true, VEC, WIDE> : quantize_kernel<T, false, VEC, WIDE>;
}
template <typename T>
void (*quantizer(int format, bool vec, bool wide))(F4QuantArgs, int) {
    return wide ? quantizer<T, true, true>(format) : vec ? quantizer<T, true, false>(format) : quantizer<T, false, false>(format);
}
template <typename T, bool VEC, int U>
void (*dequantizer(int format))(F4DequantArgs) {
    return format == BNN_F4_E8M0_32 ? dequantize_kernel<T, true, VEC, U> : dequantize_kernel<T, false, VEC, U>;
}
template <typename T>
void (*dequantizer(int format, bool vec, bool many))(F4DequantArgs) {
    if (many) return vec ? dequantizer<T, true, 4>(format) : dequantizer<T, false, 4>(format);
    return vec ? dequantizer<T, true, 1>(format) : dequantizer<T, false, 1>(format);
}

bool rows_aligned(const void* p, int dtype, int ld, int to) {
    return reinterpret_cast<uintptr_t>(p) % to == 0 && ((long long)ld * (dtype == BNN_DTYPE_F32 ? 4 : 2)) % to == 0;
}
// 1024 elements a warp where there is enough of that for every SM's warps (or too much for the grid's height), else 256.
bool long_segments(int rows, int K) {
    const int segments = ceil_div(K, 256);
    return segments > 65535 || ((long long)rows * segments >= 4LL * f4::kSms * 64 && segments >= 4);
}
// A warp's row and its columns are its block's coordinates (a division by the segments was a quarter of the instructions).
dim3 grid_of(int rows, int K, int segment) { return dim3(ceil_div(rows, WARPS), ceil_div(K, segment)); }

}  // namespace

int launch_f4_quantize(const F4QuantArgs& a, cudaStream_t st) {
    const int segment = long_segments(a.rows, a.K) ? SEGMENT : 256;
    const bool vec = rows_aligned(a.X, a.dtype, a.ldx, 16), wide = segment == SEGMENT && rows_aligned(a.X, a.dtype, a.ldx, 32);
    auto kern = a.dtype == BNN_DTYPE_F32 ? quantizer<float>(a.format, vec, wide)
              : a.dtype == BNN_DTYPE_F16 ? quantizer<__half>(a.format, vec, wide) : quantizer<__nv_bfloat16>(a.format, vec, wide);
    // (a segment always takes all scale tiles that it begins, also where K ends inside the last one)
    if (launch_pdl(kern, grid_of(a.rows, a.K, segment), dim3(WARPS * 32), 0, st, a, segment) != cudaSuccess) return BNN_ERR_CUDA;
    return launch_status();
}

int launch_f4_dequantize(const F4DequantArgs& a, cudaStream_t st) {
    const bool many = long_segments(a.rows, a.K), vec = rows_aligned(a.Y, a.dtype, a.ldy, 16);
    auto kern = a.dtype == BNN_DTYPE_F32 ? dequantizer<float>(a.format, vec, many)
              : a.dtype == BNN_DTYPE_F16 ? dequantizer<__half>(a.format, vec, many) : dequantizer<__nv_bfloat16>(a.format, vec, many);
    if (launch_pdl(kern, grid_of(a.rows, a.K, many ? 1024 : 256), dim3(WARPS * 32), 0, st, a) != cudaSuccess) return BNN_ERR_CUDA;
    return launch_status();
}

}  // namespace bnn
