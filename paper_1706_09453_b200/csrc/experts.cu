// Routing of tokens to experts, and the weighted sum of the experts' results.
//
// Router: the k largest logits of a token (ties: the lowest expert), their softmax weights, and a counting sort of the T * k
// (token, expert) pairs by expert, stable in the token: slot = offsets[expert] + how many earlier tokens chose it.  A warp takes a
// token, its logits in registers as ordered integers; a pick is a maximum over the warp.  Within a block's tokens an expert has a
// bit mask of the tokens that chose it, so that a rank is a popcount and no order of atomics can change a result.  Up to
// kOneBlock tokens one block does it all; beyond, a first kernel chooses and counts by block, and a second one adds the
// counts of the blocks before (behind a kernel that sums them, where there are many) and places.  Bound by the instructions and the
// latency of the picks, one maximum over the warp after the other: 16384 tokens, 256 experts, eight each, take 16.8 us in bf16 and 16.8 in
// fp32, 5 of them the places (the logits' 8 or 17 MB are 1.3 or 2.6; one kernel at a time and from cold caches, as a profiler runs them, choice
// and places take 16.0 and 9.6).  8 tokens, 64 experts: 3 us.  More than 512 experts are 32 logits a lane: the choice then keeps 56 to 64
// bytes a thread in local memory.
//
// A weight is expf(logit - m) / sum in fp32.  Over the chosen experts the sum adds the same expf; over all of them it adds
// 2^(x * log2 e) by the approximate instruction (fast_exp), a few 2^-22 of each term in no common direction.
//
// Weighted sum: bound by memory, 8192 tokens with four rows of 4096 bf16 each 53.5 us (6.3 TB/s).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "f4.cuh"

namespace bnn {
namespace {

constexpr int THREADS = 1024, WARPS = THREADS / 32;
constexpr int kOneBlock = 128;          // tokens
constexpr int kMaxChunk = 512;          // tokens of a block: 64 KB of masks for 1024 experts
constexpr int kManyBlocks = 160;        // from here on the counts are summed by a kernel of their own

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__half* p, float v) { *p = __float2half_rn(v); }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// fp32 -> unsigned in the same order; 0 stands for "not to be chosen" (-inf, NaN).  -0 is made +0 first: they tie.
__device__ __forceinline__ uint32_t key_of(float x) {
    if (!(x > -INFINITY)) return 0u;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    return x;
}

struct Args {
    const void* logits;
    int T, E, k, mode, chunk, words, blocks;
    long long ld;
    int32_t *index, *offsets, *slot, *source;
    float* weight;
    int row;               // E rounded up to four
    uint16_t* counts;      // [blocks][row]
    int32_t* sums;         // [blocks + 1][E], where there are many blocks
    int summed;
};

// exp(x) for x <= 0 or just above, within a few 2^-22.
__device__ __forceinline__ float fast_exp(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.44269504f));
    return r;
}

// Choices from place j on by their full keys, of the logits whose keys are at most `limit`: lane j gets the j-th one's expert (-1:
// none).  A pick is the first behind the one before it in the order of (key down, expert up).  (Short code, not at hand
// when a token in ten thousand comes here: loops that read the logits again.)
template <typename T>
__device__ __noinline__ int pick_exact(const T* x, int E, int j, int k, uint32_t limit, int expert, int lane) {
    int last = -1;
    if (lane >= j) expert = -1;
#pragma unroll 1
    for (; j < k; ++j) {
        uint32_t best = 0u;
        int at = 0x7FFFFFFF;
#pragma unroll 1
        for (int e = lane; e < E; e += 32) {
            const uint32_t key = key_of(to_f32(x[e]));
            if (key > best && (key < limit || (key == limit && e > last))) {
                best = key;
                at = e;
            }
        }
        limit = __reduce_max_sync(0xFFFFFFFFu, best);
        if (limit == 0u) break;
        last = (int)__reduce_min_sync(0xFFFFFFFFu, best == limit ? (unsigned)at : 0xFFFFFFFFu);
        if (lane == j) expert = last;
    }
    return expert;
}

__device__ __forceinline__ void keep_three(uint32_t x, uint32_t& a, uint32_t& b, uint32_t& c) {
    c = max(c, min(b, x));
    b = max(b, min(a, x));
    a = max(a, x);
}

// The same on words that hold the upper bits of a key and, in the lower ones, V - 1 - v, so that a lane's are all different and of equal
// upper bits the lowest expert comes first (across lanes: the lowest lane).  A pick is the maximum of the lanes' best
// words; the lane that had it goes on with its second and third, and looks for more only behind those.  WHOLE: the
// upper bits are all of the key that can differ.  Otherwise the answer has a bit for every pick whose upper bits are those of the
// next one, which may be before it, or (the last) of one that was not picked.
template <int V, bool WHOLE>
__device__ __forceinline__ unsigned pick_packed(const uint32_t (&word)[V], uint32_t a, uint32_t b, uint32_t c, int k, int lane, int* expert, uint32_t* picked) {
    constexpr uint32_t LOW = V - 1;            // V is a power of two
    uint32_t mine = 0u;
    int left = 3, chosen = -1;
    for (int j = 0; j < k; ++j) {
        const uint32_t most = __reduce_max_sync(0xFFFFFFFFu, a);
        if (most == 0u) break;
        const int winner = __ffs(__ballot_sync(0xFFFFFFFFu, a == most)) - 1;
        if (lane == j) {
            mine = most;
            chosen = (int)(LOW - (most & LOW)) * 32 + winner;
        }
        const bool had = lane == winner;
        a = had ? b : a;
        b = had ? c : b;
        left -= had;
        if (left == 0) {
            a = b = c = 0u;
#pragma unroll
            for (int v = 0; v < V; ++v) keep_three(word[v] < most ? word[v] : 0u, a, b, c);
            left = 3;
        }
    }
    *expert = chosen;
    *picked = mine;
    if (WHOLE) return 0u;
    const uint32_t rest = __reduce_max_sync(0xFFFFFFFFu, a);
    uint32_t next = __shfl_down_sync(0xFFFFFFFFu, mine, 1);
    if (lane == k - 1) next = rest;
    return __ballot_sync(0xFFFFFFFFu, lane < k && mine && next && (mine ^ next) <= LOW);
}

// The picks in the order of (logit down, expert up).  (A token in ten thousand comes here: short code, which is not at hand.)
__device__ __noinline__ int in_order(float x, int expert, int k, int lane) {
    int rank = 0;
#pragma unroll 1
    for (int j = 0; j < k; ++j) {
        const float y = __shfl_sync(0xFFFFFFFFu, x, j);
        const int e = __shfl_sync(0xFFFFFFFFu, expert, j);
        rank += e >= 0 && (expert < 0 || y > x || (y == x && e < expert)) ? 1 : 0;
    }
    if (expert < 0) rank = lane;
    int mine = -1;
#pragma unroll 1
    for (int j = 0; j < k; ++j) {
        const unsigned who = __ballot_sync(0xFFFFFFFFu, lane < k && rank == j);
        const int e = __shfl_sync(0xFFFFFFFFu, expert, __ffs(who) - 1);
        if (lane == j) mine = e;
    }
    return mine;
}

// A warp's token: lane j < k keeps the j-th choice (-1: none) and its weight.
template <typename T, int V>
__device__ __forceinline__ int choose(const T* x, const Args& g, int lane, float* weight) {
    float f[V];
    bool bad = false;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = v * 32 + lane;
        f[v] = e < g.E ? to_f32(x[e]) : -INFINITY;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) bad |= f[v] != f[v];
    bad = __any_sync(0xFFFFFFFFu, bad);
    uint32_t word[V], a = 0u, b = 0u, c = 0u;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const uint32_t y = __float_as_uint(f[v] + 0.0f), key = y ^ ((uint32_t)((int)y >> 31) | 0x80000000u);
        word[v] = f[v] > -INFINITY ? (key & ~(V - 1u)) | (V - 1u - v) : 0u;
        keep_three(word[v], a, b, c);
    }
    // A softmax may be taken from any point near the largest logit: that of the largest word, which is known before the picks.
    // A 16-bit type's is exact (its fp32 ends in 13 zeros: words hold the whole key).  fp32's is within 31 steps, which are less
    // than two below 2^20; beyond (finite masks, say) the first pick is taken below.
    constexpr bool WHOLE = sizeof(T) == 2;
    const uint32_t most = __reduce_max_sync(0xFFFFFFFFu, a);
    float from = most == 0u ? 0.0f : __uint_as_float((most & 0x80000000u ? most & 0x7FFFFFFFu : ~most) & ~(V - 1u));
    float total = 0.0f;
    if (g.mode == BNN_ROUTE_SOFTMAX) {
        // (the terms' errors do not add up in one direction)
#pragma unroll
        for (int v = 0; v < V; ++v) total += fast_exp(f[v] - from);
    }
    int expert = -1;
    uint32_t picked;
    const unsigned doubt = pick_packed<V, WHOLE>(word, a, b, c, g.k, lane, &expert, &picked);
    float logit = expert >= 0 ? to_f32(x[expert]) : -INFINITY;
    const bool coarse = !WHOLE && V > 1 && fabsf(from) >= 1048576.0f;
    if (doubt || coarse) {
        if (doubt >> (g.k - 1)) {
            // the last of them anew: those of the last one's upper bits
            const uint32_t upper = __shfl_sync(0xFFFFFFFFu, picked, g.k - 1) | (V - 1u);
            const int from_place = __ffs(__ballot_sync(0xFFFFFFFFu, (picked | (V - 1u)) == upper)) - 1;
            expert = pick_exact(x, g.E, from_place, g.k, upper, expert, lane);
            logit = expert >= 0 ? to_f32(x[expert]) : -INFINITY;
        }
        if (doubt & ((1u << (g.k - 1)) - 1u)) {
            expert = in_order(logit, expert, g.k, lane);
            logit = expert >= 0 ? to_f32(x[expert]) : -INFINITY;
        }
        if (coarse) {
            from = __shfl_sync(0xFFFFFFFFu, logit, 0);
            total = 0.0f;
#pragma unroll 1
            for (int e = lane; e < g.E; e += 32) total += fast_exp(to_f32(x[e]) - from);
        }
    }
    const float part = expert >= 0 ? expf(logit - from) : 0.0f;
    total = warp_sum(g.mode == BNN_ROUTE_SOFTMAX ? total : part);
    *weight = expert < 0 ? 0.0f : bad ? __uint_as_float(0x7FC00000u) : part / total;
    return expert;
}

// base[e] -> the sum of all before e, by the whole block (E <= THREADS); the sums go to `offsets` as well where it is given.
__device__ __forceinline__ void scan_experts(int* base, int E, int32_t* offsets, int lane, int warp) {
    __shared__ int whole[WARPS];
    const int e = threadIdx.x, mine = e < E ? base[e] : 0;
    int sum = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xFFFFFFFFu, sum, d);
        if (lane >= d) sum += o;
    }
    if (lane == 31) whole[warp] = sum;
    __syncthreads();
    const int before = (int)__reduce_add_sync(0xFFFFFFFFu, lane < warp ? (unsigned)whole[lane] : 0u);
    if (e < E) {
        base[e] = before + sum - mine;
        if (offsets) {
            offsets[e] = before + sum - mine;
            if (e == E - 1) offsets[E] = before + sum;
        }
    }
    __syncthreads();
}

// The places of a block's pairs; index: the block's pairs' experts (0xFFFF: none).
__device__ __forceinline__ void place(const Args& g, const uint16_t* index, const uint32_t* mask, const int* base, int first, int n) {
    for (int i = threadIdx.x; i < n * g.k; i += THREADS) {
        const int tl = i / g.k, e = index[i];
        int where = -1;
        if (e != 0xFFFF) {
            const uint32_t* m = mask + e * g.words;
            where = base[e] + __popc(m[tl >> 5] & ((1u << (tl & 31)) - 1u));
            for (int w = 0; w < tl >> 5; ++w) where += __popc(m[w]);
            g.source[where] = first + tl;
        }
        g.slot[(size_t)first * g.k + i] = where;
    }
}

// Shared memory of a block: masks [E][words], two numbers per expert, the experts of the block's pairs.
__device__ __forceinline__ int* numbers_of(uint32_t* mask, const Args& g) { return reinterpret_cast<int*>(mask + g.E * g.words); }
__device__ __forceinline__ uint16_t* pairs_of(uint32_t* mask, const Args& g) { return reinterpret_cast<uint16_t*>(mask + g.E * (g.words + 2)); }

// (The router's kernels do not let the next one start early: its blocks would wait beside the ones at work.  4096 tokens, 512 experts, eight
// each 16.6 us with a trigger at the start, 12.1 without; 8192, 64, two 11.5 and 8.4; 16384, 256, eight, with one behind the choice 27, without 16.8.)
template <typename T, int V>
__global__ void __launch_bounds__(THREADS) choose_kernel(const __grid_constant__ Args g) {
    extern __shared__ uint32_t mask[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint16_t* pairs = pairs_of(mask, g);
    for (int i = threadIdx.x; i < g.E * g.words; i += THREADS) mask[i] = 0u;
    pdl_wait();
    __syncthreads();
    const int first = blockIdx.x * g.chunk, n = min(g.chunk, g.T - first);
    for (int t = warp; t < n; t += WARPS) {
        float weight;
        const int e = choose<T, V>(static_cast<const T*>(g.logits) + (first + t) * g.ld, g, lane, &weight);
        if (lane < g.k) {
            const size_t at = (size_t)(first + t) * g.k + lane;
            g.index[at] = e;
            g.weight[at] = weight;
            pairs[t * g.k + lane] = (uint16_t)e;
            if (e >= 0) atomicOr(mask + e * g.words + (t >> 5), 1u << (t & 31));
        }
    }
    __syncthreads();
    int* base = numbers_of(mask, g);
    for (int e = threadIdx.x; e < g.row; e += THREADS) {
        int c = 0;
        if (e < g.E)
            for (int w = 0; w < g.words; ++w) c += __popc(mask[e * g.words + w]);
        if (g.blocks > 1) g.counts[(size_t)blockIdx.x * g.row + e] = (uint16_t)c;
        else if (e < g.E) base[e] = c;
    }
    if (g.blocks > 1) return;
    __syncthreads();
    scan_experts(base, g.E, g.offsets, lane, warp);
    place(g, pairs, mask, base, first, n);
}

// sums[b][e]: the counts of the blocks before b, and behind them those of all; 32 experts a block, its warps share the blocks.
__global__ void __launch_bounds__(THREADS) sum_kernel(const __grid_constant__ Args g) {
    __shared__ int part[WARPS][33];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
    const int each = ceil_div(g.blocks, WARPS), lo = min(warp * each, g.blocks), hi = min(lo + each, g.blocks);
    int sum = 0;
    if (e < g.E)
        for (int b = lo; b < hi; ++b) sum += g.counts[(size_t)b * g.row + e];
    part[warp][lane] = sum;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < warp; ++w) before += part[w][lane];
    if (e < g.E) {
        for (int b = lo; b < hi; ++b) {
            g.sums[(size_t)b * g.E + e] = before;
            before += g.counts[(size_t)b * g.row + e];
        }
        if (warp == WARPS - 1) g.sums[(size_t)g.blocks * g.E + e] = before;
    }
}

__global__ void __launch_bounds__(THREADS) place_kernel(const __grid_constant__ Args g) {
    extern __shared__ uint32_t mask[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int* base = numbers_of(mask, g);
    int* total = base + g.E;
    uint16_t* pairs = pairs_of(mask, g);
    for (int i = threadIdx.x; i < g.E * (g.words + 2); i += THREADS) mask[i] = 0u;
    pdl_wait();
    __syncthreads();
    const int first = blockIdx.x * g.chunk, n = min(g.chunk, g.T - first), mine = blockIdx.x;
    for (int i = threadIdx.x; i < n * g.k; i += THREADS) {
        const int e = g.index[(size_t)first * g.k + i], t = i / g.k;
        pairs[i] = (uint16_t)e;
        if (e >= 0) atomicOr(mask + e * g.words + (t >> 5), 1u << (t & 31));
    }
    if (g.summed) {
        for (int e = threadIdx.x; e < g.E; e += THREADS) {
            base[e] = g.sums[(size_t)mine * g.E + e];
            total[e] = g.sums[(size_t)g.blocks * g.E + e];
        }
    } else {
        // a thread of a team has four experts, teams share the blocks; integer sums, whose order is free
        const int width = g.row / 4, teams = THREADS / width, team = threadIdx.x / width, e = (threadIdx.x - team * width) * 4;
        if (team < teams) {
            int before[4] = {0, 0, 0, 0}, all[4] = {0, 0, 0, 0};
            for (int b0 = team; b0 < g.blocks; b0 += 10 * teams) {
                uint2 c[10];       // loads in flight
#pragma unroll
                for (int i = 0; i < 10; ++i) {
                    const int b = b0 + i * teams;
                    c[i] = b < g.blocks ? __ldcg(reinterpret_cast<const uint2*>(g.counts + b * g.row + e)) : make_uint2(0u, 0u);
                }
#pragma unroll
                for (int i = 0; i < 10; ++i) {
                    const int v[4] = {(int)(c[i].x & 0xFFFFu), (int)(c[i].x >> 16), (int)(c[i].y & 0xFFFFu), (int)(c[i].y >> 16)};
                    const bool earlier = b0 + i * teams < mine;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        all[q] += v[q];
                        before[q] += earlier ? v[q] : 0;
                    }
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (e + q < g.E) {
                    if (before[q]) atomicAdd(base + e + q, before[q]);
                    if (all[q]) atomicAdd(total + e + q, all[q]);
                }
        }
    }
    __syncthreads();
    scan_experts(total, g.E, mine == 0 ? g.offsets : nullptr, lane, warp);
    for (int e = threadIdx.x; e < g.E; e += THREADS) base[e] += total[e];
    __syncthreads();
    place(g, pairs, mask, base, first, n);
}

struct Plan {
    int chunk, blocks;
};
Plan plan_of(int T) {
    if (T <= kOneBlock) return {kOneBlock, 1};
    int chunk = ceil_div(T, f4::kSms);     // a block an SM, between a warp's worth of tokens and large masks
    chunk = chunk < 32 ? 32 : chunk > kMaxChunk ? kMaxChunk : chunk;
    return {chunk, ceil_div(T, chunk)};
}

template <typename T>
void (*chooser(int E))(Args) {
    if (E <= 32) return choose_kernel<T, 1>;
    if (E <= 64) return choose_kernel<T, 2>;
    if (E <= 128) return choose_kernel<T, 4>;
    if (E <= 256) return choose_kernel<T, 8>;
    if (E <= 512) return choose_kernel<T, 16>;
    return choose_kernel<T, 32>;
}

// ---- weighted sum ----
constexpr int SUM_THREADS = 128;

// Eight elements as they are loaded, and as fp32.
template <typename TZ> struct Raw { uint4 w; };
template <> struct Raw<float> { float4 a, b; };
__device__ __forceinline__ void fetch(Raw<float>& r, const float* p) {
    r.a = __ldg(reinterpret_cast<const float4*>(p));
    r.b = __ldg(reinterpret_cast<const float4*>(p) + 1);
}
template <typename TZ>
__device__ __forceinline__ void fetch(Raw<TZ>& r, const TZ* p) { r.w = __ldg(reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ void add(float (&acc)[8], float w, const Raw<float>& r) {
    const float v[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = fmaf(w, v[i], acc[i]);
}
template <typename TZ>
__device__ __forceinline__ void add(float (&acc)[8], float w, const Raw<TZ>& r) {
    const uint32_t u[4] = {r.w.x, r.w.y, r.w.z, r.w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        TZ h[2];
        memcpy(h, &u[i], 4);
        acc[2 * i] = fmaf(w, to_f32(h[0]), acc[2 * i]);
        acc[2 * i + 1] = fmaf(w, to_f32(h[1]), acc[2 * i + 1]);
    }
}
__device__ __forceinline__ void store8(float* y, const float (&acc)[8]) {
    reinterpret_cast<float4*>(y)[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    reinterpret_cast<float4*>(y)[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
}
template <typename TY>
__device__ __forceinline__ void store8(TY* y, const float (&acc)[8]) {
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        TY h[2];
        put(&h[0], acc[2 * i]);
        put(&h[1], acc[2 * i + 1]);
        memcpy(&o[i], h, 4);
    }
    *reinterpret_cast<uint4*>(y) = make_uint4(o[0], o[1], o[2], o[3]);
}

// The rows and weights of four of a token's choices; a row that does not exist is -1.
__device__ __forceinline__ void choices(const CombineArgs& g, int t, int j0, int (&s)[4], float (&w)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const size_t at = (size_t)t * g.k + j0 + j;
        s[j] = j0 + j < g.k ? __ldg(g.slot + at) : -1;
        w[j] = j0 + j < g.k ? __ldg(g.weight + at) : 0.0f;
        if (s[j] >= g.rows) s[j] = -1;
    }
}

// Block = one token and PIECES * 1024 columns; a lane has PIECES times 8 columns, and the rows of four choices are in flight at
// once.  16-byte accesses: the width is a multiple of 8.
template <typename TZ, typename TY, int PIECES>
__global__ void __launch_bounds__(SUM_THREADS) combine_kernel(const __grid_constant__ CombineArgs g, int turns) {
    pdl_trigger();
    pdl_wait();
    const int t = blockIdx.x / turns, c = ((blockIdx.x - t * turns) * PIECES * SUM_THREADS + threadIdx.x) * 8;
    if (c >= g.N) return;
    float acc[PIECES][8];
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[p][i] = 0.0f;
    const TZ* z = static_cast<const TZ*>(g.Z) + c;
    for (int j0 = 0; j0 < g.k; j0 += 4) {
        Raw<TZ> raw[4][PIECES];
        int s[4];
        float w[4];
        choices(g, t, j0, s, w);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (s[j] >= 0)
#pragma unroll
                for (int p = 0; p < PIECES; ++p)
                    if (PIECES == 1 || c + p * SUM_THREADS * 8 < g.N) fetch(raw[j][p], z + (long long)s[j] * g.ldz + p * SUM_THREADS * 8);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (s[j] >= 0)
#pragma unroll
                for (int p = 0; p < PIECES; ++p) add(acc[p], w[j], raw[j][p]);
    }
    TY* y = static_cast<TY*>(g.Y) + (long long)t * g.ldy + c;
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
        if (PIECES == 1 || c + p * SUM_THREADS * 8 < g.N) store8(y + p * SUM_THREADS * 8, acc[p]);
}

// The same element by element, for rows that start anywhere.
template <typename TZ, typename TY>
__global__ void __launch_bounds__(SUM_THREADS) combine_any_kernel(const __grid_constant__ CombineArgs g, int turns) {
    pdl_trigger();
    pdl_wait();
    const int t = blockIdx.x / turns, c0 = (blockIdx.x - t * turns) * SUM_THREADS * 8 + threadIdx.x;
    float acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0.0f;
    for (int j0 = 0; j0 < g.k; j0 += 4) {
        int s[4];
        float w[4];
        choices(g, t, j0, s, w);
        float v[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = c0 + i * SUM_THREADS;
                v[j][i] = s[j] >= 0 && c < g.N ? to_f32(static_cast<const TZ*>(g.Z)[(long long)s[j] * g.ldz + c]) : 0.0f;
            }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (s[j] >= 0)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] = fmaf(w[j], v[j][i], acc[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c0 + i * SUM_THREADS < g.N) put(static_cast<TY*>(g.Y) + (long long)t * g.ldy + c0 + i * SUM_THREADS, acc[i]);
}

template <typename TZ, typename TY>
void (*combiner(int pieces))(CombineArgs, int) {
    return pieces == 0 ? combine_any_kernel<TZ, TY> : pieces == 1 ? combine_kernel<TZ, TY, 1> : combine_kernel<TZ, TY, 2>;
}
template <typename TZ>
void (*combiner(int y_dtype, int pieces))(CombineArgs, int) {
    return y_dtype == BNN_DTYPE_F32 ? combiner<TZ, float>(pieces) : y_dtype == BNN_DTYPE_F16 ? combiner<TZ, __half>(pieces) : combiner<TZ, __nv_bfloat16>(pieces);
}

}  // namespace

size_t route_workspace_bytes(int T, int E) {
    const Plan p = plan_of(T);
    if (p.blocks == 1) return 4;
    const size_t counts = (size_t)p.blocks * ((E + 3) & ~3) * sizeof(uint16_t);
    return p.blocks < kManyBlocks ? counts : counts + (size_t)(p.blocks + 1) * E * sizeof(int32_t);
}

int launch_route(const RouteArgs& a, cudaStream_t st) {
    const Plan p = plan_of(a.T);
    Args g{};
    g.logits = a.logits; g.T = a.T; g.E = a.E; g.k = a.k; g.mode = a.mode; g.ld = a.ld;
    g.chunk = p.chunk; g.words = ceil_div(p.chunk, 32); g.blocks = p.blocks;
    g.index = a.index; g.offsets = a.offsets; g.slot = a.slot; g.source = a.source; g.weight = a.weight;
    g.row = (a.E + 3) & ~3;
    g.counts = static_cast<uint16_t*>(a.workspace);
    g.sums = reinterpret_cast<int32_t*>(g.counts + (size_t)p.blocks * g.row);
    g.summed = p.blocks >= kManyBlocks;
    auto smem_of = [](int E, int words, int pairs) { return E * (words + 2) * (int)sizeof(uint32_t) + pairs * (int)sizeof(uint16_t); };
    const int smem = smem_of(a.E, g.words, p.chunk * a.k), most = smem_of(f4::kMaxGroups, kMaxChunk / 32, kMaxChunk * 32);
    void (*choose)(Args) = a.dtype == BNN_DTYPE_F32 ? chooser<float>(a.E) : a.dtype == BNN_DTYPE_F16 ? chooser<__half>(a.E) : chooser<__nv_bfloat16>(a.E);
    if (!ensure_dynamic_smem(reinterpret_cast<const void*>(choose), most) ||
        (p.blocks > 1 && !ensure_dynamic_smem(reinterpret_cast<const void*>(place_kernel), most)))
        return BNN_ERR_CUDA;
    if (launch_pdl(choose, dim3(p.blocks), dim3(THREADS), smem, st, g) != cudaSuccess) return BNN_ERR_CUDA;
    if (p.blocks > 1) {
        if (g.summed && launch_pdl(sum_kernel, dim3(ceil_div(a.E, 32)), dim3(THREADS), 0, st, g) != cudaSuccess) return BNN_ERR_CUDA;
        if (launch_pdl(place_kernel, dim3(p.blocks), dim3(THREADS), smem, st, g) != cudaSuccess) return BNN_ERR_CUDA;
    }
    return launch_status();
}

int launch_combine(const CombineArgs& a, cudaStream_t st) {
    const int zs = a.dtype == BNN_DTYPE_F32 ? 4 : 2, ys = a.y_dtype == BNN_DTYPE_F32 ? 4 : 2;
    const bool vec = a.N % 8 == 0 && aligned16(a.Z) && aligned16(a.Y) && ((long long)a.ldz * zs) % 16 == 0 && ((long long)a.ldy * ys) % 16 == 0;
    // Two pieces a lane where that leaves every SM a few blocks.
    const int pieces = !vec ? 0 : a.N > SUM_THREADS * 8 && (long long)a.T * ceil_div(a.N, SUM_THREADS * 16) >= f4::kSms * 8 ? 2 : 1;
    const int turns = ceil_div(a.N, SUM_THREADS * 8 * (pieces == 2 ? 2 : 1));
    if ((long long)a.T * turns > 0x7FFFFFFF) return BNN_ERR_SHAPE;
    void (*kern)(CombineArgs, int) = a.dtype == BNN_DTYPE_F32 ? combiner<float>(a.y_dtype, pieces)
                                   : a.dtype == BNN_DTYPE_F16 ? combiner<__half>(a.y_dtype, pieces) : combiner<__nv_bfloat16>(a.y_dtype, pieces);
    if (launch_pdl(kern, dim3((unsigned)(a.T * turns)), dim3(SUM_THREADS), 0, st, a, turns) != cudaSuccess) return BNN_ERR_CUDA;
    return launch_status();
}

}  // namespace bnn
