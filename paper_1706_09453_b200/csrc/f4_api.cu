// extern "C" boundary of the operators on 4-bit floating point and on experts: argument validation.  No allocation, no sync.
#include <limits.h>
#include <math.h>

#include <type_traits>
#include <utility>

#include "f4.cuh"

using namespace bnn;

namespace {

constexpr int kMaxExponent = 64, kMaxChoices = 32;
// Rows, tokens and columns are rounded up to whole blocks (4096 columns at most) in 32 bits.
constexpr int kMaxLength = 0x7FFFFFFF - 4096;

bool known_format(int f) { return f == BNN_F4_E8M0_32 || f == BNN_F4_E4M3_16; }
bool known_dtype(int d) { return d == BNN_DTYPE_F32 || d == BNN_DTYPE_F16 || d == BNN_DTYPE_BF16; }
bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
size_t size_of(int dtype) { return dtype == BNN_DTYPE_F32 ? 4 : 2; }

long long tiles_of(int format, long long rows, int groups, int K) {
    return (rows / 128 + groups) * (long long)f4::scale_tiles(format, K);
}

// Stored form of a quantised matrix.
int check_f4(const void* codes, int ld, const void* scales, size_t scale_bytes, int format, long long rows, int groups, int K) {
    if (!codes || !scales) return BNN_ERR_NULL;
    if (ld < f4::code_bytes(K)) return BNN_ERR_SHAPE;
    if (ld % 16 || !aligned16(codes) || !aligned16(scales)) return BNN_ERR_ALIGN;
    const long long tiles = tiles_of(format, rows, groups, K);
    if (tiles > 0x7FFFFFFF) return BNN_ERR_SHAPE;
    if (scale_bytes < (size_t)tiles * 512) return BNN_ERR_WORKSPACE;
    return BNN_OK;
}

int check_groups(const int32_t* offsets, int groups) {
    if (groups < 1 || groups > f4::kMaxGroups || (!offsets && groups != 1)) return BNN_ERR_SHAPE;
    return offsets && !aligned_to(offsets, 4) ? BNN_ERR_ALIGN : BNN_OK;
}

int gemm_checked(const void* a, int lda, const void* a_scales, size_t a_scale_bytes, const int32_t* offsets, int groups,
                 const void* w, int ldw, const void* w_scales, size_t w_scale_bytes, int M, int N, int K, int format, int exponent,
                 void* Y, int dtype, int ldy, const bnn_epilogue* epi, void* stream) {
    if (!known_format(format)) return BNN_ERR_UNSUPPORTED;
    if (M < 1 || N < 1 || K < 1 || K > f4::kMaxK) return BNN_ERR_SHAPE;
    if (exponent < -kMaxExponent || exponent > kMaxExponent) return BNN_ERR_SHAPE;
    if (int rc = check_groups(offsets, groups)) return rc;
    const long long units = (long long)groups * N;
    if (units > 0x7FFFFFFF - 256 || M > kMaxLength) return BNN_ERR_SHAPE;
    if (((long long)M / 32 + groups) * ceil_div(N, 128) > 0x7FFF0000) return BNN_ERR_SHAPE;
    if (int rc = check_f4(a, lda, a_scales, a_scale_bytes, format, M, groups, K)) return rc;
    if (int rc = check_f4(w, ldw, w_scales, w_scale_bytes, format, units, groups, K)) return rc;
    F4GemmArgs g{};
    g.act = BNN_ACT_NONE;
    if (epi) {
        g.act = epi->act;
        g.sign_mode = epi->sign_mode;
        g.scale = epi->scale;
        g.shift = epi->shift;
        if (!aligned_to(g.scale, 4) || !aligned_to(g.shift, 4)) return BNN_ERR_ALIGN;
    }
    if (g.act == BNN_ACT_SIGN_PACK) {
        if (Y) return BNN_ERR_UNSUPPORTED;
        if (!epi->out_bits) return BNN_ERR_NULL;
        if (epi->ldob < words_for(N)) return BNN_ERR_SHAPE;
        if (epi->ldob % 4 || !aligned16(epi->out_bits)) return BNN_ERR_ALIGN;
        if (g.sign_mode != BNN_SIGN_ZERO_POS && g.sign_mode != BNN_SIGN_ZERO_NEG) return BNN_ERR_UNSUPPORTED;
        g.out_bits = epi->out_bits;
        g.ldob = epi->ldob;
    } else {
        if (g.act != BNN_ACT_NONE && g.act != BNN_ACT_HARDTANH && g.act != BNN_ACT_SIGMOID) return BNN_ERR_UNSUPPORTED;
        if (epi && epi->out_bits) return BNN_ERR_UNSUPPORTED;      // bits are written by BNN_ACT_SIGN_PACK alone
        if (!known_dtype(dtype)) return BNN_ERR_UNSUPPORTED;
        if (!Y) return BNN_ERR_NULL;
        if (ldy < N) return BNN_ERR_SHAPE;
        if (!aligned_to(Y, size_of(dtype))) return BNN_ERR_ALIGN;
    }
    g.a = static_cast<const uint8_t*>(a); g.lda = lda; g.a_scales = static_cast<const uint8_t*>(a_scales);
    g.offsets = offsets; g.groups = groups;
    g.w = static_cast<const uint8_t*>(w); g.ldw = ldw; g.w_scales = static_cast<const uint8_t*>(w_scales);
    g.M = M; g.N = N; g.K = K; g.format = format; g.factor = ldexpf(1.0f, exponent);
    g.Y = Y; g.dtype = dtype; g.ldy = ldy;
    return launch_f4_gemm(g, static_cast<cudaStream_t>(stream));
}

// A call whose arguments come as words.
template <typename T>
bool fits(int64_t w) { return !std::is_same<T, int>::value || (w >= INT_MIN && w <= INT_MAX); }
template <typename T>
T from_word(int64_t w) {
    if constexpr (std::is_pointer<T>::value) return reinterpret_cast<T>(static_cast<uintptr_t>(w));
    else return static_cast<T>(w);
}
template <typename... Args, size_t... I>
int call_words(int (*f)(Args...), const int64_t* w, std::index_sequence<I...>) {
    if (!(fits<Args>(w[I]) && ...)) return BNN_ERR_SHAPE;
    return f(from_word<Args>(w[I])...);
}
template <typename... Args>
int call_words(int (*f)(Args...), const int64_t* w, int n) {
    return n == (int)sizeof...(Args) ? call_words(f, w, std::index_sequence_for<Args...>()) : BNN_ERR_SHAPE;
}

}  // namespace

extern "C" {

int bnn_call_words(int call, const int64_t* words, int n) {
    if (!words) return BNN_ERR_NULL;
    switch (call) {
        case BNN_CALL_F4_QUANTIZE: return call_words(bnn_f4_quantize, words, n);
        case BNN_CALL_F4_DEQUANTIZE: return call_words(bnn_f4_dequantize, words, n);
        case BNN_CALL_F4_GEMM: return call_words(bnn_f4_gemm, words, n);
        case BNN_CALL_F4_GEMM_GROUPED: return call_words(bnn_f4_gemm_grouped, words, n);
        case BNN_CALL_ROUTE_EXPERTS: return call_words(bnn_route_experts, words, n);
        case BNN_CALL_COMBINE_EXPERTS: return call_words(bnn_combine_experts, words, n);
        default: return BNN_ERR_UNSUPPORTED;
    }
}

int bnn_f4_pitch(int K) { return K < 1 || K > f4::kMaxK ? 0 : f4::code_bytes(K); }

size_t bnn_f4_scale_bytes(int format, int rows, int K, int groups) {
    if (!known_format(format) || rows < 1 || K < 1 || K > f4::kMaxK || groups < 1 || groups > f4::kMaxGroups) return 0;
    return (size_t)tiles_of(format, rows, groups, K) * 512;
}

int bnn_f4_quantize(const void* X, int dtype, int src_rows, int K, int ldx, const int32_t* source, const int32_t* offsets, int groups,
                    int rows, int format, int exponent, void* codes, int ldc, void* scales, size_t scale_bytes, void* stream) {
    if (!X) return BNN_ERR_NULL;
    if (!known_format(format) || !known_dtype(dtype)) return BNN_ERR_UNSUPPORTED;
    if (rows < 1 || rows > kMaxLength || src_rows < 1 || K < 1 || K > f4::kMaxK || ldx < K || (!source && src_rows < rows)) return BNN_ERR_SHAPE;
    if (exponent < -kMaxExponent || exponent > kMaxExponent) return BNN_ERR_SHAPE;
    if (int rc = check_groups(offsets, groups)) return rc;
    if (int rc = check_f4(codes, ldc, scales, scale_bytes, format, rows, groups, K)) return rc;
    if (!aligned_to(X, size_of(dtype)) || !aligned_to(source, 4)) return BNN_ERR_ALIGN;
    F4QuantArgs a{};
    a.X = X; a.dtype = dtype; a.src_rows = src_rows; a.ldx = ldx; a.source = source; a.offsets = offsets; a.groups = groups;
    a.rows = rows; a.K = K; a.format = format; a.factor = ldexpf(1.0f, exponent);
    a.codes = static_cast<uint8_t*>(codes); a.ldc = ldc; a.scales = static_cast<uint8_t*>(scales);
    return launch_f4_quantize(a, static_cast<cudaStream_t>(stream));
}

int bnn_f4_dequantize(const void* codes, int ldc, const void* scales, size_t scale_bytes, const int32_t* offsets, int groups, int rows,
                      int K, int format, int exponent, void* Y, int dtype, int ldy, void* stream) {
    if (!Y) return BNN_ERR_NULL;
    if (!known_format(format) || !known_dtype(dtype)) return BNN_ERR_UNSUPPORTED;
    if (rows < 1 || rows > kMaxLength || K < 1 || K > f4::kMaxK || ldy < K) return BNN_ERR_SHAPE;
    if (exponent < -kMaxExponent || exponent > kMaxExponent) return BNN_ERR_SHAPE;
    if (int rc = check_groups(offsets, groups)) return rc;
    if (int rc = check_f4(codes, ldc, scales, scale_bytes, format, rows, groups, K)) return rc;
    if (!aligned_to(Y, size_of(dtype))) return BNN_ERR_ALIGN;
    F4DequantArgs a{};
    a.codes = static_cast<const uint8_t*>(codes); a.ldc = ldc; a.scales = static_cast<const uint8_t*>(scales);
    a.offsets = offsets; a.groups = groups; a.rows = rows; a.K = K; a.format = format; a.factor = ldexpf(1.0f, exponent);
    a.Y = Y; a.dtype = dtype; a.ldy = ldy;
    return launch_f4_dequantize(a, static_cast<cudaStream_t>(stream));
}

int bnn_f4_gemm(const void* A, int lda, const void* a_scales, size_t a_scale_bytes, const void* W, int ldw, const void* w_scales,
                size_t w_scale_bytes, int M, int N, int K, int format, int exponent, void* Y, int dtype, int ldy,
                const bnn_epilogue* epi, void* stream) {
    return gemm_checked(A, lda, a_scales, a_scale_bytes, nullptr, 1, W, ldw, w_scales, w_scale_bytes, M, N, K, format, exponent,
                        Y, dtype, ldy, epi, stream);
}

int bnn_f4_gemm_grouped(const void* A, int lda, const void* a_scales, size_t a_scale_bytes, const int32_t* offsets, int groups,
                        const void* W, int ldw, const void* w_scales, size_t w_scale_bytes, int M, int N, int K, int format,
                        int exponent, void* Y, int dtype, int ldy, const bnn_epilogue* epi, void* stream) {
    if (!offsets) return BNN_ERR_NULL;
    return gemm_checked(A, lda, a_scales, a_scale_bytes, offsets, groups, W, ldw, w_scales, w_scale_bytes, M, N, K, format, exponent,
                        Y, dtype, ldy, epi, stream);
}

int bnn_f4_gemm_form(int M, int N, int K, int groups, int sms, bnn_f4_form* form) {
    if (!form) return BNN_ERR_NULL;
    if (M < 1 || M > kMaxLength || N < 1 || N > 0x7FFFFFFF - 256 || K < 1 || K > f4::kMaxK || groups < 0 || groups > f4::kMaxGroups || sms < 0)
        return BNN_ERR_SHAPE;
    return f4_gemm_form(M, N, K, groups, sms, form);
}

size_t bnn_route_workspace_bytes(int T, int E) {
    return T < 1 || T > kMaxLength || E < 1 || E > f4::kMaxGroups ? 0 : route_workspace_bytes(T, E);
}

int bnn_route_experts(const void* logits, int dtype, int T, int E, int ld, int k, int mode, int32_t* index, float* weight,
                      int32_t* offsets, int32_t* slot, int32_t* source, void* workspace, size_t workspace_bytes, void* stream) {
    if (!logits || !index || !weight || !offsets || !slot || !source) return BNN_ERR_NULL;
    if (!known_dtype(dtype) || (mode != BNN_ROUTE_SOFTMAX && mode != BNN_ROUTE_SOFTMAX_CHOSEN)) return BNN_ERR_UNSUPPORTED;
    if (T < 1 || T > kMaxLength || E < 1 || E > f4::kMaxGroups || ld < E || k < 1 || k > E || k > kMaxChoices || T > 0x7FFFFFFF / k) return BNN_ERR_SHAPE;
    if (!aligned_to(logits, size_of(dtype)) || !aligned_to(index, 4) || !aligned_to(weight, 4) || !aligned_to(offsets, 4) ||
        !aligned_to(slot, 4) || !aligned_to(source, 4) || !aligned16(workspace))
        return BNN_ERR_ALIGN;
    if (!workspace || workspace_bytes < route_workspace_bytes(T, E)) return BNN_ERR_WORKSPACE;
    RouteArgs a{};
    a.logits = logits; a.dtype = dtype; a.T = T; a.E = E; a.ld = ld; a.k = k; a.mode = mode;
    a.index = index; a.weight = weight; a.offsets = offsets; a.slot = slot; a.source = source; a.workspace = workspace;
    return launch_route(a, static_cast<cudaStream_t>(stream));
}

int bnn_combine_experts(const void* Z, int z_dtype, int rows, int ldz, const int32_t* slot, const float* weight, int T, int k, int N,
                        void* Y, int y_dtype, int ldy, void* stream) {
    if (!Z || !slot || !weight || !Y) return BNN_ERR_NULL;
    if (!known_dtype(z_dtype) || !known_dtype(y_dtype)) return BNN_ERR_UNSUPPORTED;
    if (rows < 1 || T < 1 || k < 1 || k > kMaxChoices || N < 1 || N > kMaxLength || ldz < N || ldy < N) return BNN_ERR_SHAPE;
    if (!aligned_to(Z, size_of(z_dtype)) || !aligned_to(Y, size_of(y_dtype)) || !aligned_to(slot, 4) || !aligned_to(weight, 4))
        return BNN_ERR_ALIGN;
    CombineArgs a{};
    a.Z = Z; a.dtype = z_dtype; a.rows = rows; a.ldz = ldz; a.slot = slot; a.weight = weight; a.T = T; a.k = k; a.N = N;
    a.Y = Y; a.y_dtype = y_dtype; a.ldy = ldy;
    return launch_combine(a, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
