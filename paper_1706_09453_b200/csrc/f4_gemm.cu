// Product of two quantised matrices, dense or by groups of rows (experts), on the block-scaled 4-bit tensor-core path:
//   Y[m][n] = act(2^e * scale[n] * sum_k a[m][k] w[n][k] + shift[n]),  a and w: e2m1 codes times their blocks' scales.
//
// The units (rows of W) are the MMA's M side and the activations' rows its N side: an N can be any multiple of 16, so a tile's
// width follows the rows that a group has, down to a single token, while 128 units always fill the M side.  The accumulator then
// has a unit in each lane, and a warp stores 32 consecutive units of a row.
//
// Roles of a CTA: one thread copies the stages (256 positions of K: 128 bytes of each row of codes, and their scale tiles)
// with TMA, one warp moves the scales to tensor memory (tcgen05.cp) and issues the MMAs, eight warps empty the accumulator.
// Two accumulators alternate.  Tiles of 256 columns leave 512 - 2 * 256 = 0 columns for the scales, so these accumulators
// overlap by 32 columns, which the epilogue reads first: the next tile starts as soon as they are read.
//
// Bound by the bytes that an SM takes in from L2: 42.5 a clock, which plain loads reach as well.  A step of a pair (256 units x 256
// rows x 256 of K) is 36 KB, 843 clocks, for 512 of MMA; without any MMA 8192 x 4096 x 4096 takes 49.7 us instead of 52.9.  On top come
// the stores (without them 97 us instead of 106 at 8192 x 4096 x 8192, 5.2 PFLOP/s; that is at the full clock, as replayed from a graph in short
// runs: back to back under the power limit the same product takes 125 us, 4.4 PFLOP/s) and, where K is short, the epilogue, 5200 clocks a
// tile.  Each TMA instruction costs as well: two copies of 64 rows and scale tiles one by one instead of one copy per operand were 118
// us instead of 109.  e4m3 scales, of which there are twice as many, take 112.  Scale copies to tensor memory cost nothing measurable.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "f4.cuh"
#include "tcgen05.cuh"

namespace bnn {
namespace {

using namespace tc;

constexpr int BM = 128;                  // units of a CTA's tile
constexpr int BK_BYTES = 128;            // bytes of codes of a row in a stage
constexpr int BK = 256;
constexpr int EPI_WARPS = 8, TMA_WARP = 8, MMA_WARP = 9, THREADS = 320;
constexpr int TMEM_COLS = 512, SF_COL = 480;
constexpr int PANEL = 8;
constexpr int SMEM_LIMIT = 232448, MAX_STAGES = 10;
constexpr int OUT_CHUNK = 32 * 64;       // a warp's 32 rows x 32 units of 16 bits on their way out
constexpr int PAIR_ROWS = 256;           // rows of a pair's tile
constexpr int MAX_SPLIT = 4;             // CTAs that share the K of a tile

template <bool MX, bool PAIR, int TN, bool SPLIT>
struct Shape {
    static constexpr int KATOMS = MX ? 2 : 4;                     // scale tiles (four blocks of K) of a stage
    static constexpr int B_ROWS = PAIR ? TN / 2 : TN;             // rows of activations in this CTA's shared memory
    static constexpr int ROW_TILES = TN > 128 ? 2 : 1;            // scale tiles across the activations' rows
    static constexpr int A_BYTES = BM * BK_BYTES, B_BYTES = B_ROWS * BK_BYTES;
    static constexpr int SFA_BYTES = KATOMS * 512, SFB_BYTES = ROW_TILES * KATOMS * 512;
    static constexpr int STAGE = A_BYTES + B_BYTES + SFA_BYTES + SFB_BYTES;
    static constexpr int CONTROL = 512 + (f4::kMaxGroups + 1) * 8;
    static constexpr int OUT_BYTES = SPLIT ? TN * BM * 4 : EPI_WARPS * OUT_CHUNK;
    static constexpr int FIT = (SMEM_LIMIT - 1024 - CONTROL - OUT_BYTES) / STAGE;
    static constexpr int STAGES = FIT > MAX_STAGES ? MAX_STAGES : FIT;
    static constexpr int SMEM = STAGES * STAGE + OUT_BYTES + CONTROL + 1024;
    static constexpr int ACC_STEP = TN > 224 ? SF_COL - TN : TN;  // second accumulator's first column
    static constexpr int OVERLAP = ACC_STEP < TN ? TN - ACC_STEP : 0;
    static_assert(STAGE % 1024 == 0 && STAGES >= 3 && ACC_STEP + TN <= SF_COL && (OVERLAP == 0 || OVERLAP == 32) && SMEM <= SMEM_LIMIT, "");
};

struct Maps {
    CUtensorMap w, a, w_scales, a_scales;
};

struct Args {
    const int32_t* offsets;
    int groups, M, N, K, kt;
    float factor;
    const float* scale;
    const float* shift;
    int act, sign_mode, box, split, tile_rows;
    int early;              // the next kernel may start while this one runs
    void* Y;
    int dtype, pieces;
    long long ldy;
    uint32_t* out_bits;
    long long ldob;
    TcStatus status;
};

template <int A> struct Act { static constexpr int value = A; };

struct Control {
    uint64_t full[MAX_STAGES], empty[MAX_STAGES], acc_full, acc_free, drained;
    WaitState wait;
    uint32_t tmem_base;
    int first[f4::kMaxGroups + 1];      // first row of each group, held inside 0 .. M
    int tiles[f4::kMaxGroups + 1];      // row tiles of all groups before
};
static_assert(sizeof(Control) <= 512 + (f4::kMaxGroups + 1) * 8, "");

struct Tile {
    int g, row0, n, unit0, a_tile;
    uint32_t sf_off;        // columns of the scale tile before the first row's
};

// The group of which row tile j (of all groups, counted one behind the other) is one: the last whose tiles start at or before it.
__device__ __forceinline__ int group_of(const Control* ctl, int groups, int j) {
    int lo = 0, hi = groups;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (ctl->tiles[mid] <= j) lo = mid; else hi = mid;
    }
    return lo;
}
__device__ __forceinline__ Tile make_tile(const Control* ctl, int tile_rows, int group, int row_tile, int unit0) {
    Tile t;
    t.g = group;
    t.unit0 = unit0;
    const int off = row_tile * tile_rows, begin = ctl->first[group];
    t.row0 = begin + off;
    t.n = min(tile_rows, ctl->first[group + 1] - t.row0);
    t.a_tile = begin / 128 + group + off / 128;
    t.sf_off = (off & 127) >> 5;
    return t;
}

// Tile number w: panels of PANEL unit tiles, in which the units run fastest, so that the tiles that run at the same time
// are about as many unit tiles as row tiles and share both operands' reads.  (Consecutive tiles for a CTA, whose weights then stay
// in shared memory, are slower: 8192 x 4096 x 8192 113 us instead of 108, 32 groups 89 instead of 83.)
__device__ __forceinline__ Tile tile_at(const Control* ctl, const Args& g, int w, int unit_tiles, int unit_step) {
    const int rows = ctl->tiles[g.groups], panel = w / (rows * PANEL), in = w - panel * rows * PANEL;
    const int wide = min(PANEL, unit_tiles - panel * PANEL), j = in / wide, group = group_of(ctl, g.groups, j);
    return make_tile(ctl, g.tile_rows, group, j - ctl->tiles[group], (panel * PANEL + in - j * wide) * unit_step);
}

template <bool PAIR>
__device__ __forceinline__ int columns_of(int n) { return PAIR ? (n + 31) & ~31 : (n + 15) & ~15; }

__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__half* p, float v) { *p = __float2half_rn(v); }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

template <int ACT>
__device__ __forceinline__ float activate(float v) {
    if (ACT == BNN_ACT_HARDTANH) return v != v ? v : fminf(fmaxf(v, -1.0f), 1.0f);
    if (ACT == BNN_ACT_SIGMOID) return 1.0f / (1.0f + expf(-v));
    return v;
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __half) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Where a warp's chunk of 32 units x 32 rows goes: the first unit's address in the first row, how many units and rows exist.
struct Chunk {
    long long ldy;
    int units, rows;
};

// A lane has a unit, a store 32 consecutive ones of a row: fp32, and 16 bits where rows start anywhere.
template <int ACT, typename T, typename F>
__device__ __forceinline__ void store_units(T* y, const Chunk& c, uint32_t taddr, int lane, float scale, float shift, F&& read) {
    uint32_t acc[32];
    tmem_ld32(taddr, acc);
    tmem_ld_wait();
    read();
    if (lane >= c.units) return;
    y += lane;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        if (i < c.rows) put(y, activate<ACT>(fmaf(scale, __uint_as_float(acc[i]), shift)));
        y += c.ldy;
    }
}

// 16 bits, rows of Y on 16-byte boundaries: the accumulator comes in the layout of an MMA's result, goes to shared memory
// transposed and from there, in pieces of 16 bytes, out in rows of 256 bytes: the four warps that hold the tile's 128 units share a
// chunk of 32 rows.  (8192 x 1024 x 8192: element by element 88 us, a warp's rows of 64 bytes 46 us.)
// out: the four warps' 32 x 256 bytes; piece p of row r lies at r * 256 + 16 * (p ^ r % 8), so that neither side meets itself in a
// bank.  scale, shift: of units lane / 4 + 8 i.  c.units: from the tile's first unit on.  `next`: the chunk to load into acc once
// this one's values are taken.
struct Frag {
    uint32_t lo[16], hi[16];
    __device__ __forceinline__ void load(uint32_t taddr) {
        tmem_ld_frag32(taddr, lo);
        tmem_ld_frag32(taddr + (16u << 16), hi);
    }
};
template <int ACT, typename T>
__device__ __forceinline__ void store_pieces(T* y, const Chunk& c, Frag& acc, int half, int quarter, int lane, uint32_t out,
                                             const float (&scale)[4], const float (&shift)[4], bool more, uint32_t next) {
    uint32_t v[4][4];
    auto val = [&](uint32_t a, int i) { return activate<ACT>(fmaf(scale[i], __uint_as_float(a), shift[i])); };
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j][0] = pack2(val(acc.lo[4 * j], 0), val(acc.lo[4 * j + 1], 0), T());
        v[j][1] = pack2(val(acc.lo[4 * j + 2], 1), val(acc.lo[4 * j + 3], 1), T());
        v[j][2] = pack2(val(acc.hi[4 * j], 2), val(acc.hi[4 * j + 1], 2), T());
        v[j][3] = pack2(val(acc.hi[4 * j + 2], 3), val(acc.hi[4 * j + 3], 3), T());
    }
    if (more) acc.load(next);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = 8 * j + (lane & 7);
        stmatrix4_trans(out + row * 256 + ((quarter * 4 + (lane >> 3)) ^ (row & 7)) * 16, v[j][0], v[j][1], v[j][2], v[j][3]);
    }
    bar_sync_128(4 + half);
    const int piece = lane & 15, units = c.units - piece * 8;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = 8 * quarter + 2 * j + (lane >> 4);
        const uint4 w = lds128u(out + row * 256 + (piece ^ (row & 7)) * 16);
        if (row >= c.rows) continue;
        T* p = y + row * c.ldy + piece * 8;
        if (units >= 8) {
            *reinterpret_cast<uint4*>(p) = w;
        } else {
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < units) reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)(u[i >> 1] >> (16 * (i & 1)));
        }
    }
    bar_sync_128(4 + half);
}

template <bool MX, bool PAIR, int TN, bool SPLIT>
__device__ __forceinline__ void body(const Maps& maps, const Args& g) {
    using S = Shape<MX, PAIR, TN, SPLIT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    constexpr int OUT_AT = S::STAGES * S::STAGE;
    Control* ctl = reinterpret_cast<Control*>(smem + OUT_AT + S::OUT_BYTES);
    volatile int* abort_flag = &ctl->wait.abort;
    if (g.early) pdl_trigger();
    const int warp = warp_index(), lane = threadIdx.x & 31;
    const int rank = PAIR ? (int)cluster_rank() : 0, part = SPLIT ? (int)cluster_rank() : 0;
    constexpr int CTAS = PAIR ? 2 : 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) {
            mbar_init(smem_u32(&ctl->full[s]), 1);      // (rank 0:) its copying thread, and the bytes of both CTAs
            mbar_init(smem_u32(&ctl->empty[s]), 1);     // a commit
        }
        mbar_init(smem_u32(&ctl->acc_full), 1);
        mbar_init(smem_u32(&ctl->drained), 1);
        mbar_init(smem_u32(&ctl->acc_free), CTAS * EPI_WARPS);
        wait_state_init(&ctl->wait, g.status);
        mbar_init_fence();
    }
    __syncwarp();
    if (warp == MMA_WARP) {
        if constexpr (PAIR) {
            tmem_alloc_pair(smem_u32(&ctl->tmem_base), TMEM_COLS);
        } else {
            tmem_alloc(smem_u32(&ctl->tmem_base), TMEM_COLS);
            tmem_relinquish();
        }
    }
    pdl_wait();
    // Groups.  Offsets that make no sense are held inside the matrix and made to ascend, so that no row is in two groups.
    if (g.offsets) {
        for (int i = threadIdx.x; i <= g.groups; i += THREADS) ctl->first[i] = min(max(__ldg(g.offsets + i), 0), g.M);
        __syncthreads();
        if (warp == 0) {
            int most = 0, before = 0;
            for (int i0 = 0; i0 <= g.groups; i0 += 32) {
                const int i = i0 + lane, lowest = most;
                int first = i <= g.groups ? ctl->first[i] : 0;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int o = __shfl_up_sync(0xFFFFFFFFu, first, d);
                    if (lane >= d) first = max(first, o);
                }
                first = max(first, lowest);
                if (i <= g.groups) ctl->first[i] = first;
                most = __shfl_sync(0xFFFFFFFFu, first, 31);
                // tiles of group i - 1
                int prev = __shfl_up_sync(0xFFFFFFFFu, first, 1);
                if (lane == 0) prev = lowest;
                int sum = i > 0 && i <= g.groups ? (first - prev + g.tile_rows - 1) / g.tile_rows : 0;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int o = __shfl_up_sync(0xFFFFFFFFu, sum, d);
                    if (lane >= d) sum += o;
                }
                if (i <= g.groups) ctl->tiles[i] = before + sum;
                before += __shfl_sync(0xFFFFFFFFu, sum, 31);
            }
        }
    } else if (threadIdx.x == 0) {
        ctl->first[0] = 0;
        ctl->first[1] = g.M;
        ctl->tiles[0] = 0;
        ctl->tiles[1] = ceil_div(g.M, g.tile_rows);
    }
    tc_fence_before_sync();
    __syncthreads();
    if constexpr (PAIR || SPLIT) cluster_sync();     // the others have started
    tc_fence_after_sync();
    const uint32_t tmem = ctl->tmem_base;

    const int unit_tiles = ceil_div(g.N, BM * CTAS), nks = ceil_div(g.K, BK);
    const int total = ctl->tiles[g.groups] * unit_tiles;
    // this CTA's (pair's) tiles; with SPLIT a cluster has one tile at most, and a CTA its share of the steps of K
    const int workers = gridDim.x / (SPLIT ? g.split : CTAS), worker = blockIdx.x / (SPLIT ? g.split : CTAS);
    const int k0 = SPLIT ? nks * part / g.split : 0, k1 = SPLIT ? nks * (part + 1) / g.split : nks;

    int issued = 0;                      // steps that the copying thread has asked for
    if (warp == TMA_WARP) {
        if (lane == 0) {
            int s = 0;
            uint32_t ph = 1;
            bool ok = true;
            for (int w = worker; w < total && ok; w += workers) {
                const Tile t = tile_at(ctl, g, w, unit_tiles, BM * CTAS);
                const int cols = columns_of<PAIR>(t.n);
                const int mine = PAIR ? cols / 2 : cols, boxes = ceil_div(mine, g.box);
                const int unit = t.unit0 + rank * BM, row = t.row0 + rank * mine;
                const int w_row = t.g * g.N + unit;
                const int w_tile = (int)((long long)t.g * g.N / 128) + t.g + unit / 128;
                const uint32_t bytes = S::A_BYTES + boxes * g.box * BK_BYTES + S::SFA_BYTES + S::SFB_BYTES;
                for (int ks = k0; ks < k1; ++ks) {
                    ok = mbar_wait(smem_u32(&ctl->empty[s]), ph, abort_flag);
                    if (!ok) break;
                    const uint32_t a = smem_u32(smem) + s * S::STAGE, b = a + S::A_BYTES, sf = b + S::B_BYTES;
                    const uint32_t bar = smem_u32(&ctl->full[s]), bar0 = PAIR ? peer_addr(bar, 0) : bar;
                    if (rank == 0) mbar_arrive_expect_tx(bar, CTAS * bytes);
                    ++issued;
                    auto load = [&](uint32_t to, const CUtensorMap* map, int x, int y) {
                        if constexpr (PAIR) tma_load_2d_pair(to, map, x, y, bar0);
                        else tma_load_2d(to, map, x, y, bar);
                    };
                    auto load_scales = [&](uint32_t to, const CUtensorMap* map, int katom, int tile) {
                        if constexpr (PAIR) tma_load_3d_pair(to, map, 0, katom, tile, bar0);
                        else tma_load_3d(to, map, 0, katom, tile, bar);
                    };
                    load(a, &maps.w, ks * BK_BYTES, w_row);
                    for (int i = 0; i < boxes; ++i) load(b + i * g.box * BK_BYTES, &maps.a, ks * BK_BYTES, row + i * g.box);
                    load_scales(sf, &maps.w_scales, ks * S::KATOMS, w_tile);
                    load_scales(sf + S::SFA_BYTES, &maps.a_scales, ks * S::KATOMS, t.a_tile);
                    if (++s == S::STAGES) { s = 0; ph ^= 1u; }
                }
            }
        }
        __syncwarp();
    } else if (warp == MMA_WARP) {
        int s = 0, buf = 0;
        uint32_t ph = 0, pfree = 1;       // a fresh barrier passes parity 1
        bool ok = rank == 0;
        for (int w = worker; w < total && ok; w += workers) {
            const Tile t = tile_at(ctl, g, w, unit_tiles, BM * CTAS);
            const int cols = columns_of<PAIR>(t.n);
            const uint32_t id0 = instr_desc_f4(BM * CTAS, cols, MX, 0), id2 = instr_desc_f4(BM * CTAS, cols, MX, MX ? 2 : 0);
            // the accumulator before this one is read as far as this one overlaps it, and all of the one before that
            ok = warp_wait(smem_u32(&ctl->acc_free), pfree, abort_flag, lane);
            if (!ok) break;
            pfree ^= 1u;
            tc_fence_after_sync();
            const uint32_t d = tmem + buf * S::ACC_STEP, sfa = tmem + SF_COL, sfb = sfa + 8, sfo = t.sf_off;
            for (int ks = k0; ks < k1; ++ks) {
                ok = warp_wait(smem_u32(&ctl->full[s]), ph, abort_flag, lane);
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t a = smem_u32(smem) + s * S::STAGE, b = a + S::A_BYTES, sf = b + S::B_BYTES;
                const uint64_t da = smem_desc_sw128(a), db = smem_desc_sw128(b);
                const int left = g.K - ks * BK;
                if (elect_one()) {
                    // Halves of 128 positions: their scales, then two MMAs of 64.  The copies and MMAs of one thread run in
                    // order, so the same columns hold the scales of every half.
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (h * 128 >= left) break;
#pragma unroll
                        for (int c = 0; c < S::KATOMS / 2; ++c) {
                            const int katom = h * (S::KATOMS / 2) + c;
                            tmem_copy_scales<PAIR>(sfa + 4 * c, sf + katom * 512);
#pragma unroll
                            for (int r = 0; r < S::ROW_TILES; ++r)
                                tmem_copy_scales<PAIR>(sfb + 4 * S::ROW_TILES * c + 4 * r, sf + S::SFA_BYTES + (r * S::KATOMS + katom) * 512);
                        }
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            if (h * 128 + m * 64 >= left) break;
                            const int x = (h * 2 + m) * 2;       // 32 bytes, in units of 16
                            mma_f4<MX, PAIR>(d, da + x, db + x, MX && m ? id2 : id0, MX ? sfa : sfa + 4 * m,
                                             (MX ? sfb : sfb + 4 * S::ROW_TILES * m) + sfo, ks != k0 || h != 0 || m != 0);
                        }
                    }
                    if constexpr (PAIR) mma_commit_pair(smem_u32(&ctl->empty[s]));
                    else mma_commit(smem_u32(&ctl->empty[s]));
                }
                if (++s == S::STAGES) { s = 0; ph ^= 1u; }
            }
            if (ok && elect_one()) {
                if constexpr (PAIR) mma_commit_pair(smem_u32(&ctl->acc_full));
                else mma_commit(smem_u32(&ctl->acc_full));
            }
            buf ^= 1;
        }
        __syncwarp();
    } else if constexpr (SPLIT) {
        // this part's sums to shared memory, [row][unit]
        const int half = warp >> 2, quarter = warp & 3;
        if (worker < total) {
            const Tile t = tile_at(ctl, g, worker, unit_tiles, BM);
            if (warp_wait_relaxed(smem_u32(&ctl->acc_full), 0u, abort_flag, lane)) {
                tc_fence_after_sync();
                float* sums = reinterpret_cast<float*>(smem + OUT_AT) + quarter * 32 + lane;
#pragma unroll 1
                for (int at = half; at * 32 < t.n; at += 2) {
                    uint32_t acc[32];
                    tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + at * 32, acc);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (at * 32 + j < t.n) sums[(at * 32 + j) * BM] = __uint_as_float(acc[j]);
                }
            }
        }
    } else {
        const int half = warp >> 2, quarter = warp & 3;
        const uint32_t free0 = PAIR ? peer_addr(smem_u32(&ctl->acc_free), 0) : smem_u32(&ctl->acc_free);
        const uint32_t out = smem_u32(smem) + OUT_AT + half * 4 * OUT_CHUNK;
        uint32_t pfull = 0;
        int buf = 0;
        for (int w = worker; w < total; w += workers) {
            const Tile t = tile_at(ctl, g, w, unit_tiles, BM * CTAS);
            const int u0 = t.unit0 + rank * BM + quarter * 32, chunks = ceil_div(t.n, 32);
            // per-unit affine: of the lane's unit, or (16-bit results) of units lane / 4 + 8 i
            const bool pieces = g.pieces;
            const size_t p = (size_t)t.g * g.N + u0;
            float scale[4], shift[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int u = pieces ? (lane >> 2) + 8 * i : lane;
                scale[i] = (g.scale && u0 + u < g.N ? __ldg(g.scale + p + u) : 1.0f) * g.factor;
                shift[i] = g.shift && u0 + u < g.N ? __ldg(g.shift + p + u) : 0.0f;
            }
            // (the four warps of a half take the same decision: they meet at barriers below)
            const bool ok = warp_wait_relaxed(smem_u32(&ctl->acc_full), pfull, abort_flag, lane);
            if (!(half ? epi_all_b(ok) : epi_all(ok))) break;
            pfull ^= 1u;
            tc_fence_after_sync();
            const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * S::ACC_STEP);
            bool freed = false;
            auto read = [&] {
                if (freed) return;
                freed = true;
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (PAIR) mbar_arrive_cluster(free0);
                    else mbar_arrive(free0);
                }
            };
            // the columns that the next tile's accumulator overlaps come first: the highest of the first one, the lowest
            // of the second
            const int mine = (chunks - half + 1) >> 1;
            Chunk c{g.ldy, g.N - u0, 0};
            auto chunk_at = [&](int i) { return half + 2 * (buf == 0 ? mine - 1 - i : i); };
            auto by_pieces = [&](auto* y, auto act) {
                Frag acc;
                acc.load(taddr + chunk_at(0) * 32);
                Chunk whole{g.ldy, g.N - t.unit0 - rank * BM, 0};
#pragma unroll 1
                for (int i = 0; i < mine; ++i) {
                    const int at = chunk_at(i);
                    whole.rows = min(32, t.n - at * 32);
                    tmem_ld_wait();
                    read();
                    store_pieces<decltype(act)::value>(y + (t.row0 + at * 32) * g.ldy + t.unit0 + rank * BM, whole, acc, half, quarter, lane, out,
                                                       scale, shift, i + 1 < mine, taddr + chunk_at(i + 1) * 32);
                }
            };
            auto by_units = [&](auto* y, auto act) {
#pragma unroll 1
                for (int i = 0; i < mine; ++i) {
                    const int at = chunk_at(i);
                    c.rows = min(32, t.n - at * 32);
                    store_units<decltype(act)::value>(y + (t.row0 + at * 32) * g.ldy + u0, c, taddr + at * 32, lane, scale[0], shift[0], read);
                }
            };
            auto typed = [&](auto act) {
                if (g.dtype == BNN_DTYPE_F32) by_units(static_cast<float*>(g.Y), act);
                else if (g.dtype == BNN_DTYPE_F16) pieces ? by_pieces(static_cast<__half*>(g.Y), act) : by_units(static_cast<__half*>(g.Y), act);
                else pieces ? by_pieces(static_cast<__nv_bfloat16*>(g.Y), act) : by_units(static_cast<__nv_bfloat16*>(g.Y), act);
            };
            if (mine > 0) {
                if (g.out_bits) {
#pragma unroll 1
                    for (int i = 0; i < mine; ++i) {
                        const int at = chunk_at(i);
                        uint32_t acc[32], word = 0;
                        tmem_ld32(taddr + at * 32, acc);
                        tmem_ld_wait();
                        read();
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const float v = fmaf(scale[0], __uint_as_float(acc[j]), shift[0]);
                            const uint32_t b = __ballot_sync(0xFFFFFFFFu, lane < c.units && sign_is_pos(v, g.sign_mode));
                            if (lane == j) word = b;
                        }
                        if (lane < t.n - at * 32 && c.units > 0) g.out_bits[(t.row0 + at * 32 + lane) * g.ldob + (u0 >> 5)] = word;
                    }
                } else if (g.act == BNN_ACT_NONE) {
                    typed(Act<BNN_ACT_NONE>());
                } else if (g.act == BNN_ACT_HARDTANH) {
                    typed(Act<BNN_ACT_HARDTANH>());
                } else {
                    typed(Act<BNN_ACT_SIGMOID>());
                }
            }
            read();
            buf ^= 1;
        }
    }

    if constexpr (SPLIT) {
        // every CTA adds up its share of the rows from all parts, a warp a row and a lane four units, in the order of K: a row's
        // sum must not depend on whose share it falls into
        __syncwarp();
        cluster_sync();
        if (warp < EPI_WARPS && worker < total) {
            const Tile t = tile_at(ctl, g, worker, unit_tiles, BM);
            const int per = ceil_div(t.n, g.split), end = min((part + 1) * per, t.n), unit = t.unit0 + lane * 4, units = g.N - unit;
            const size_t p = (size_t)t.g * g.N + unit;
            float scale[4], shift[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                scale[i] = (g.scale && i < units ? __ldg(g.scale + p + i) : 1.0f) * g.factor;
                shift[i] = g.shift && i < units ? __ldg(g.shift + p + i) : 0.0f;
            }
            for (int r = part * per + warp; r < end; r += EPI_WARPS) {
                const uint32_t at = smem_u32(smem) + OUT_AT + (r * BM + lane * 4) * 4;
                float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
                for (int i = 0; i < g.split; ++i) {
                    const float4 x = ld_cluster4(peer_addr(at, i));
                    v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
                }
                uint32_t bits = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = fmaf(scale[i], v[i], shift[i]);
                    bits |= (i < units && sign_is_pos(v[i], g.sign_mode) ? 1u : 0u) << ((lane & 7) * 4 + i);
                    v[i] = g.act == BNN_ACT_HARDTANH ? activate<BNN_ACT_HARDTANH>(v[i]) : g.act == BNN_ACT_SIGMOID ? activate<BNN_ACT_SIGMOID>(v[i]) : v[i];
                }
                const long long row = t.row0 + r;
                if (g.out_bits) {
#pragma unroll
                    for (int d = 1; d < 8; d <<= 1) bits |= __shfl_xor_sync(0xFFFFFFFFu, bits, d);
                    if (!(lane & 7) && units > 0) g.out_bits[row * g.ldob + (unit >> 5)] = bits;
                } else {
                    const long long to = row * g.ldy + unit;
                    if (g.dtype != BNN_DTYPE_F32 && g.pieces && units >= 4) {
                        const uint2 w = g.dtype == BNN_DTYPE_F16 ? make_uint2(pack2(v[0], v[1], __half()), pack2(v[2], v[3], __half()))
                                                                 : make_uint2(pack2(v[0], v[1], __nv_bfloat16()), pack2(v[2], v[3], __nv_bfloat16()));
                        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(g.Y) + to) = w;
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (i >= units) break;
                            if (g.dtype == BNN_DTYPE_F32) put(static_cast<float*>(g.Y) + to + i, v[i]);
                            else if (g.dtype == BNN_DTYPE_F16) put(static_cast<__half*>(g.Y) + to + i, v[i]);
                            else put(static_cast<__nv_bfloat16*>(g.Y) + to + i, v[i]);
                        }
                    }
                }
            }
        }
        __syncwarp();
        cluster_sync();          // nobody reads this CTA's sums any more
    }

    // every thread arrives here, also after a wait that ran out
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) {
        // What is still on its way ends first, whatever the limit was that ran out: the MMAs, and the copies.  Those of a pair are counted on rank
        // 0, which may have stopped before it asked for as many as rank 1: rank 1, which cannot see that barrier, gives its own the time.  (A
        // rank that did not give up has seen its last accumulator, and so the end of all copies.)
        const long long until = clock64() + kDrainClocks;
        if (warp == MMA_WARP) {
            if (rank == 0 && elect_one()) {
                if constexpr (PAIR) mma_commit_pair(smem_u32(&ctl->drained));
                else mma_commit(smem_u32(&ctl->drained));
            }
            __syncwarp();
            mbar_wait_out(smem_u32(&ctl->drained), 0u, until);
        } else if (warp == TMA_WARP && lane == 0) {
            if (rank == 0) {
                for (int i = max(0, issued - S::STAGES); i < issued; ++i)
                    mbar_wait_out(smem_u32(&ctl->full[i % S::STAGES]), (uint32_t)(i / S::STAGES) & 1u, until);
            } else {
                while (issued > 0 && clock64() < until) {}
            }
        }
        __syncwarp();
        __syncthreads();
    }
    if constexpr (PAIR) cluster_sync();
    if (warp == MMA_WARP) {
        tc_fence_after_sync();
        if constexpr (PAIR) tmem_dealloc_pair(tmem, TMEM_COLS);
        else tmem_dealloc(tmem, TMEM_COLS);
    }
    if (threadIdx.x == 0 && ctl->wait.abort) atomicExch(g.status.word, 1);
}

template <bool MX, int TN, bool SPLIT>
__global__ void __launch_bounds__(THREADS, 1) f4_gemm_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Args g) {
    body<MX, false, TN, SPLIT>(maps, g);
}

// The same on pairs of CTAs: 256 units x up to 256 rows, half of the rows in the shared memory of each.
template <bool MX>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
f4_gemm_pair_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Args g) {
    body<MX, true, PAIR_ROWS, false>(maps, g);
}

template <typename S>
bool encode_maps(Maps* m, const F4GemmArgs& a, int kt, int box) {
    const int bytes = f4::code_bytes(a.K);
    const long long units = (long long)a.groups * a.N;
    return encode_code_map(&m->w, a.w, a.ldw, units, bytes, BM) && encode_code_map(&m->a, a.a, a.lda, a.M, bytes, box) &&
           encode_scale_map(&m->w_scales, a.w_scales, units / 128 + a.groups, kt, 1, S::KATOMS) &&
           encode_scale_map(&m->a_scales, a.a_scales, f4::row_tiles(a.M, a.groups), kt, S::ROW_TILES, S::KATOMS);
}

// The sizes that a form is chosen by; groups 0: a dense matrix.
struct Sizes {
    int M, N, K, groups;
};

// An upper bound on the tiles of a form: the groups' rows are only known on the device.  n rows make at most (n + rows - 1) / rows tiles, and
// at most min(M, groups) groups have any.  Of a dense matrix it is the number itself.
long long tiles_of(const Sizes& z, int rows, int units) {
    const long long live = !z.groups ? 1 : z.M < z.groups ? z.M : z.groups;
    return (z.M + live * (rows - 1)) / rows * ceil_div(z.N, units);
}

// How a product is cut up: tiles of ctas * 128 units x tile_rows rows (of `width` in the kernel's layout), copied `box` rows at a time, their K
// shared by `split` CTAs.
struct Form {
    int ctas, tile_rows, width, box, split;
};

// Up to 32 rows: clusters of 2 or 4 CTAs share a tile's K where the tiles alone leave SMs idle.  (Quantisation and product, one row,
// us without and with: K = N = 2048 6.9 and 6.3, 4096 10.0 and 7.7, 8192 15.6 and 12.2, K = 8192 N = 2048 15.2 and 8.8; the product alone
// on 31 or 32 rows: 5.5, 6.6, 11.9 and 7.6, and on 33, which do without: 5.8, 8.5, 14.5 and 13.8.  Clusters of 8
// wait for so many free SMs of a GPC that they lose: 10.4 at 2048.  So does adding up 128 rows and more: 256 rows of 2048 8.2 and 11.5.)
Form few_rows(const Sizes& z, int sms) {
    const long long tiles = tiles_of(z, 32, BM);
    int split = 1;
    while (split < MAX_SPLIT && tiles * split * 2 <= sms && split * 2 <= ceil_div(z.K, BK)) split *= 2;
    return {1, 32, 32, z.M <= 16 ? 16 : 32, split};
}

// Which form.  Up to 32 rows: tiles of 32 (a group's second tile of 32 would start inside a tile of scales, so that these are 32
// rows in all).  Else single CTAs (128 units x 128 rows), pairs of 256 units x 256 rows, or, without groups, of 192 rows (every second tile then
// starts in the middle of a tile of scales), by the clocks that the SMs are estimated to take: the turns, what each takes as measured on
// many turns (the epilogue's time where K is short), and the last one's epilogue.  Measured, us single / 192 / 256: 1024 rows, K = N =
// 2048 6.8 / 8.0 / 8.1; 731 rows, N = 3307 11.1 / 9.0 / 9.4; 2048 rows 11.0 / 11.3 / 8.6; 4096 x 4096 x 4096 47.3 / 36.6 / 31.5; 4096 x 512 x
// 4096 16.4 / 15.3 / 14.6; 16384 rows by 32 groups of 2048 x 4096 118 / 90 / 80.  (Pairs of 128 rows win nowhere.)
// Groups of less than 128 rows on average are bound by their weights' bytes, and narrow tiles have more of them on their way: 2048
// rows by 32 groups 19.3 and 21.2.
Form form_of(const Sizes& z, int sms) {
    if (z.M <= 32) return few_rows(z, sms);
    const int rows = z.groups ? ceil_div(z.M, z.groups) : z.M;      // of a group, on average
    const long long steps = ceil_div(z.K, BK);
    auto clocks = [&](int tile, int ctas, long long shortest, long long step, long long more, long long last) {
        // (half a tile for the rest of each group)
        const long long row_tiles = z.groups ? z.M / tile + (z.groups + 1) / 2 : ceil_div(z.M, tile);
        const long long turns = (row_tiles * ceil_div(z.N, BM * ctas) + sms / ctas - 1) / (sms / ctas), turn = steps * step + more;
        return turns * (turn > shortest ? turn : shortest) + last;
    };
    if (rows >= 128 && sms >= 2) {
        const long long single = clocks(128, 1, 3500, 753, 1450, 1900), high = clocks(256, 2, 5200, 743, 2350, 3800);
        const long long low = z.groups ? high : clocks(192, 2, 3900, 700, 2200, 3000);
        if (low < high && low < single) return {2, 192, PAIR_ROWS, 96, 1};
        if (high < single) return {2, 256, PAIR_ROWS, 128, 1};
    }
    return {1, 128, 128, rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128, 1};
}

Sizes sizes_of(const F4GemmArgs& a) { return {a.M, a.N, a.K, a.offsets ? a.groups : 0}; }

template <bool MX, bool PAIR, int TN, bool SPLIT>
int launch_form(const F4GemmArgs& a, Args g, const Form& f, int sms, cudaStream_t st) {
    using S = Shape<MX, PAIR, TN, SPLIT>;
    constexpr int CTAS = PAIR ? 2 : 1;
    Maps maps;
    g.box = f.box;
    g.tile_rows = f.tile_rows;
    g.split = f.split;
    void (*kern)(Maps, Args);
    if constexpr (PAIR) kern = f4_gemm_pair_kernel<MX>;
    else kern = f4_gemm_kernel<MX, TN, SPLIT>;
    if (!ensure_dynamic_smem(reinterpret_cast<const void*>(kern), S::SMEM) || !encode_maps<S>(&maps, a, g.kt, f.box)) return BNN_ERR_CUDA;
    const long long tiles = tiles_of(sizes_of(a), f.tile_rows, BM * CTAS);
    // The next kernel's blocks beside this one's are worth it where every SM has one tile at most (one token 5.2 us, and 5.6 where
    // they come at the end); beside many turns they only get in each other's way (quantisation and product, 8192 x 2048 x 2048: 29.4, and
    // 27.6 at the end).
    g.early = tiles <= sms / CTAS;
    if constexpr (SPLIT) {
        if (launch_pdl_cluster(kern, dim3((unsigned)(tiles * g.split)), dim3(THREADS), g.split, S::SMEM, st, maps, g) != cudaSuccess) return BNN_ERR_CUDA;
    } else {
        const int grid = CTAS * (int)(tiles < sms / CTAS ? tiles : sms / CTAS);
        if (launch_pdl(kern, dim3(grid), dim3(THREADS), S::SMEM, st, maps, g) != cudaSuccess) return BNN_ERR_CUDA;
    }
    return launch_status();
}

template <bool MX>
int launch_format(const F4GemmArgs& a, const Args& g, int sms, cudaStream_t st) {
    const Form f = form_of(sizes_of(a), sms);
    if (f.ctas == 2) return launch_form<MX, true, PAIR_ROWS, false>(a, g, f, sms, st);
    if (f.width == 128) return launch_form<MX, false, 128, false>(a, g, f, sms, st);
    return f.split > 1 ? launch_form<MX, false, 32, true>(a, g, f, sms, st) : launch_form<MX, false, 32, false>(a, g, f, sms, st);
}

}  // namespace

int f4_gemm_form(int M, int N, int K, int groups, int sms, bnn_f4_form* form) {
    if (sms == 0) sms = device_sm_count();
    if (sms < 1) return BNN_ERR_CUDA;
    const Form f = form_of({M, N, K, groups}, sms);
    form->ctas = f.ctas;
    form->rows = f.tile_rows;
    form->split = f.split;
    return BNN_OK;
}

int launch_f4_gemm(const F4GemmArgs& a, cudaStream_t st) {
    const int sms = device_sm_count();
    Args g{};
    g.offsets = a.offsets; g.groups = a.groups; g.M = a.M; g.N = a.N; g.K = a.K;
    g.kt = f4::scale_tiles(a.format, a.K);
    g.factor = a.factor; g.scale = a.scale; g.shift = a.shift; g.act = a.act; g.sign_mode = a.sign_mode;
    g.Y = a.Y; g.dtype = a.dtype; g.ldy = a.ldy;
    g.pieces = a.Y && a.dtype != BNN_DTYPE_F32 && aligned16(a.Y) && a.ldy % 8 == 0;
    g.out_bits = a.out_bits; g.ldob = a.ldob;
    g.status = tc_status();
    if (sms < 1 || !g.status.word) return BNN_ERR_CUDA;
    return a.format == BNN_F4_E8M0_32 ? launch_format<true>(a, g, sms, st) : launch_format<false>(a, g, sms, st);
}

}  // namespace bnn
