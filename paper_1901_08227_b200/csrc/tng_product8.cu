// Products of 8-bit codes with scales for each row of either side:
//   out[i][j] = (float(sum_l a[i][l] b[j][l]) sa[i]) sb[j] + bias[j].
//
// The int32 sums are exact, so every variant below gives the same bits whatever order it sums in.
//
// Every wait on a barrier has a poll limit.  When one runs out the sums are incomplete: the outputs that the CTAs concerned
// still owe become NaN (`ok`, `good` below), which is how a call that never waits for the GPU reports it.
#include <math_constants.h>

#include "tng_codes.cuh"
#include "tng_umma.cuh"

namespace tng {
namespace {

// A sum as an output, each operation one fp32 rounding.
__device__ __forceinline__ float scaled(int acc, float sa, float sb, bool has_bias, float bias) {
    const float v = __fmul_rn(__fmul_rn((float)acc, sa), sb);
    return has_bias ? __fadd_rn(v, bias) : v;
}

// ---- a linear layer of at most 8 tokens in one launch: the weights are streamed past them -------------------
// Bound by reading b once (from memory: 1 x 4096 x 4096 bf16 6.5 us, 8 x 16384 x 2048 11.4 us, launches included).  Every CTA codes the
// tokens itself while its first weights travel, one group of registers a thread: at most 16384 elements with the tokens
// counted as a power of two.  (Codes by a launch of their own and the tensor-memory kernel below: 9.3 and 12.7 us, and
// 3.5 us more of the host's time; 8 x 512 x 512 3.3 us against 5.3.)  The tokens' codes stay in shared memory; a CTA goes over tiles of sixteen rows of b, KS warps
// sharing a tile along the contraction, 256 codes a warp and step: a lane has every fourth 16 bytes of two rows, eight
// loads of them, the next step's issued before this one's are used.  A warp-wide m16n8k32 instruction takes the weights as
// its 16 rows straight from the loaded words and the tokens as its 8 columns: the contraction may run in any order as
// long as both sides agree, so a lane's 16 consecutive codes serve as its words of two instructions.  These instructions are
// slow here (270 cycles where one waits for another, hence four chains; byte products on the integer pipe took 7 cycles
// each, three times as long at 8 tokens), but they keep up with memory.
constexpr int kStreamThreads = 256, kStreamTokens = 8, kStreamHold = 8;
__host__ __device__ inline uint32_t stream_pitch(uint64_t k) { return (uint32_t)((k + 255) / 256 * 256 + 64); }   // 64 mod 128: no bank conflicts
// Threads a token while its line is coded: all 256 over the tokens' next power of two.
__host__ __device__ inline uint32_t stream_share(uint64_t tokens) { return kStreamThreads / (tokens > 4 ? 8 : tokens > 2 ? 4 : tokens > 1 ? 2 : 1); }

__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The tokens' codes and scales into shared memory, zero up to the pitch.
template <typename X>
__device__ __forceinline__ void stream_tokens(const X* x, uint64_t ldx, uint32_t tokens, uint32_t k, int8_t* codes, uint32_t pitch,
                                              float* scales, uint32_t* part) {
    const uint32_t groups = (k + 7) / 8, all = pitch / 8;
    // (at most kStreamHold groups of eight a thread: all loads at once)
    const uint32_t share = stream_share(tokens), t = threadIdx.x / share, lane = threadIdx.x & (share - 1);
    const X* row = x + (uint64_t)(t < tokens ? t : 0) * ldx;
    const bool vec = aligned16(row) && k % 8 == 0;
    Raw8<X> v[kStreamHold];
    uint32_t m = 0;
    if (vec) {
#pragma unroll
        for (int h = 0; h < kStreamHold; ++h) v[h] = lane + h * share < groups ? load_raw8(row + (lane + h * share) * 8) : zero_raw8<X>();
    } else {
#pragma unroll
        for (int h = 0; h < kStreamHold; ++h)
            v[h] = lane + h * share < groups ? fetch_raw8<X, false>(row, (lane + h * share) * 8, k) : zero_raw8<X>();
    }
#pragma unroll
    for (int h = 0; h < kStreamHold; ++h) m = top_raw8<X>(v[h], m);
    m = __reduce_max_sync(kFullMask, top_bits<X>(top_of_halves<X>(m)));
    if (share > 32) {
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
        __syncthreads();
        const uint32_t w = share >> 5;
        for (uint32_t i = 0; i < w; ++i) m = max(m, part[t * w + i]);
    }
    if (t < tokens) {
        const LineScale s = line_scale(m);
        if (lane == 0) scales[t] = s.scale;
        uint2* dst = reinterpret_cast<uint2*>(codes + t * pitch);
#pragma unroll
        for (int h = 0; h < kStreamHold; ++h) {
            const uint32_t g = lane + h * share;
            if (g >= all) break;
            float f[8];
            widen8(v[h], f);
            dst[g] = code8<false>(f, s.inv, DrawArgs{}, DrawRow{}, 0);
        }
        for (uint32_t g = lane + kStreamHold * share; g < all; g += share) dst[g] = make_uint2(0u, 0u);
    }
}

template <typename T>
__global__ void __launch_bounds__(kStreamThreads, 2) product8_stream_kernel(const T* x, uint64_t ldx, const __grid_constant__ Product8 p) {
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ float scales[kStreamTokens];
    __shared__ uint32_t part[8];
    __shared__ int red[2][8][kStreamTokens][17];           // [half][warp][token][row]
    int8_t* codes = reinterpret_cast<int8_t*>(dyn);
    const uint32_t k = (uint32_t)p.k, pitch = stream_pitch(k), kparts = (k + 255) / 256, tokens = (uint32_t)p.m;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const uint32_t ks = kparts >= 5 ? 8u : kparts >= 3 ? 4u : kparts;          // warps sharing a tile
    const uint32_t per_round = 8 / ks, sub = warp / ks, kp0 = warp & (ks - 1), chans = per_round * 16;
    const uint32_t steps = (kparts + ks - 1) / ks;          // of 256 codes, for a warp that has the most
    const uint64_t rounds = ((p.n + 15) / 16 + per_round - 1) / per_round;
    const uint64_t mine = blockIdx.x < rounds ? (rounds - 1 - blockIdx.x) / gridDim.x + 1 : 0;

    uint4 buf[8];                                           // [four chunks][row g, row g + 8]
    const auto load = [&](uint64_t round, uint32_t step) {
        const uint64_t row = (round * per_round + sub) * 16 + g;
        const uint32_t c = (kp0 + step * ks) * 256 + q * 16;
        const int8_t *src = p.b + row * p.ldb + c, *src8 = src + 8 * p.ldb;
        if (row + 8 < p.n && c + 192 < k) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                buf[2 * i] = load16_once(src + 64 * i);
                buf[2 * i + 1] = load16_once(src8 + 64 * i);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
                buf[2 * i] = row < p.n && c + 64 * i < k ? load16_once(src + 64 * i) : zero;
                buf[2 * i + 1] = row + 8 < p.n && c + 64 * i < k ? load16_once(src8 + 64 * i) : zero;
            }
        }
    };
    grid_wait();
    grid_go();
    if (mine) load(blockIdx.x, 0);
    stream_tokens<T>(x, ldx, tokens, k, codes, pitch, scales, part);
    __syncthreads();

    T* out = static_cast<T*>(p.out);
    for (uint64_t j = 0; j < mine; ++j) {
        const uint64_t round = blockIdx.x + j * gridDim.x;
        const uint64_t first = round * chans + threadIdx.x % chans;     // the channel of this thread's outputs (chans divides 256)
        const float sb = first < p.n ? load_f32(p.sb + first) : 0.f, bias = first < p.n && p.bias ? load_f32(p.bias + first) : 0.f;
        int acc[4][4] = {};
        for (uint32_t step = 0; step < steps; ++step) {
            uint4 w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = buf[i];
            if (step + 1 < steps) load(round, step + 1);
            else if (j + 1 < mine) load(round + gridDim.x, 0);
            const uint32_t c = (kp0 + step * ks) * 256 + q * 16;
            if (kp0 + step * ks < kparts) {
                uint4 a[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    a[i] = g < tokens ? *reinterpret_cast<const uint4*>(codes + g * pitch + c + 64 * i) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    mma_s8(acc[(2 * i) & 3], w[2 * i].x, w[2 * i + 1].x, w[2 * i].y, w[2 * i + 1].y, a[i].x, a[i].y);
                    mma_s8(acc[(2 * i + 1) & 3], w[2 * i].z, w[2 * i + 1].z, w[2 * i].w, w[2 * i + 1].w, a[i].z, a[i].w);
                }
            }
        }
        int(*mem)[kStreamTokens][17] = red[j & 1];
#pragma unroll
        for (int e = 0; e < 4; ++e)                         // element e: row g (+ 8 from 2 on), token 2 q + (e & 1)
            mem[warp][2 * q + (e & 1)][g + (e & 2) * 4] = (acc[0][e] + acc[1][e]) + (acc[2][e] + acc[3][e]);
        __syncthreads();                                    // the other half of `red` is free: its readers passed this barrier last round
        for (uint32_t i = threadIdx.x; i < chans * tokens; i += kStreamThreads) {
            if (first >= p.n) break;
            const uint32_t tok = i / chans, ch = i - tok * chans;
            int a = 0;
            for (uint32_t s = 0; s < ks; ++s) a += mem[(ch >> 4) * ks + s][tok][ch & 15];
            out[(uint64_t)tok * p.ldo + first] = from_f32<T>(scaled(a, scales[tok], sb, p.bias, bias));
        }
    }
}

// ---- pairs of CTAs: 256 x 256 outputs a tile ------------------------------------------------------------
// Two CTAs (two SMs) work on one tile: each holds 128 rows of a and 128 rows of b per stage, and the matrix
// instruction of the even CTA reads both shared memories (8192^3, bf16 out: 318 to 334 us, 3290 TOP/s and up, the tensor pipe 88% busy;
// 390 us once the power limit holds the clock); the accumulators are 128 rows x 256 columns in each
// CTA's tensor memory, twice, so that one tile is written out while the next is summed.  A stage of 128 codes
// takes 513 cycles where the instruction rate allows 512 (measured with the feed running); 256 x 128 tiles take 470
// for half the work, so small outputs split the contraction instead of the tile:
// SPLIT: a cluster of S pairs takes S consecutive parts of one tile's contraction; pair q then adds the others' int32
// sums, read from their shared memories, to its own for 256/S of the columns and writes those out.
// Warps: 0-15 write out (a quarter of the rows and of the columns each: with eight the last tile's output took 3 us), 16
// feeds, 17 issues.
constexpr int kPairThreads = 576;
constexpr uint32_t kPairTile = 256;
constexpr uint32_t kStageStride = 2048;                    // staging of one warp
constexpr uint32_t kPairStages = 6, kPairHalf = 128 * 128, kPairStage = 2 * kPairHalf;
static_assert(128 * kPairTile * 4 <= kPairStages * kPairStage, "the stages also hold the sums");
constexpr uint32_t kPairSmem = 1024 + kPairStages * kPairStage + 16 * kStageStride + 256;

// What one launch computes: one product, or two independent ones (a gradient's dx and dw, which together leave fewer
// pairs idle at the end than one after the other).
struct PairArgs {
    Product8 p[2];
};
struct PairMaps {
    CUtensorMap a, b, o;
};

// A pair's tiles, the same sequence for each of its roles.  Within a product: groups of eight tile rows, columns outside.
// Of two products the one with the longer contraction (job `first`) goes first, tile by tile over the pairs; the pairs that
// get one tile of it less then take as many of the other's as that is worth, and the rest goes over all pairs again.
struct TileWalk {
    struct Job {
        uint32_t tiles_m, tiles_n, kblocks;
    } job[2];
    uint32_t first, pair, pairs, spare, extra, phase, next, cur, tm, tn;

    __device__ __forceinline__ static Job shape(const Product8& p) { return {(uint32_t)((p.m + 255) / 256), (uint32_t)((p.n + 255) / 256), (uint32_t)((p.k + 127) / 128)}; }
    __device__ __forceinline__ uint32_t count(uint32_t j) const { return job[j].tiles_m * job[j].tiles_n; }
    template <bool DUAL> __device__ __forceinline__ void start(const PairArgs& args, uint32_t pair_, uint32_t pairs_) {
        pair = pair_;
        pairs = pairs_;
        job[0] = shape(args.p[0]);
        if (DUAL) job[1] = shape(args.p[1]);
        first = DUAL && job[1].kblocks > job[0].kblocks;
        phase = 0;
        next = pair;
        spare = extra = 0;
        if (DUAL) {
            spare = count(first) % pairs;                  // pairs with one more of the first job's tiles
            const uint32_t worth = spare ? job[first].kblocks / job[first ^ 1].kblocks : 0;
            const uint32_t all = worth * (pairs - spare), have = count(first ^ 1);
            extra = all < have ? all : have;
        }
    }
    // The next tile into cur (job), tm, tn; false when there is none.
    template <bool DUAL> __device__ __forceinline__ bool step() {
        uint32_t t = next;
        cur = first;
        if (phase == 0) {
            if (t < count(first)) {
                next = t + pairs;
            } else if (!DUAL) {
                return false;
            } else {
                phase = 1;
                next = pair >= spare ? pair - spare : extra;
            }
        }
        if (DUAL && phase == 1) {
            cur = first ^ 1;
            t = next;
            if (t < extra) {
                next = t + (pairs - spare);
            } else {
                phase = 2;
                next = extra + (pair >= spare ? pair - spare : pair + pairs - spare);
            }
        }
        if (DUAL && phase == 2) {
            cur = first ^ 1;
            t = next;
            if (t >= count(cur)) return false;
            next = t + pairs;
        }
        const Job& j = job[cur];
        const uint32_t per = 8 * j.tiles_n, g = t / per, top = g * 8;
        const uint32_t rows = j.tiles_m - top < 8 ? j.tiles_m - top : 8, r = t - g * per;
        tn = r / rows;
        tm = top + (r - tn * rows);
        return true;
    }
};

// A lane's column scale and bias of a chunk of 32 columns; fetched before the sums are waited for.
struct ColumnScale {
    float sb, bias;
};
__device__ __forceinline__ ColumnScale column_scale(const Product8& p, uint64_t col) {
    const bool in = col < p.n;
    return {in ? load_f32(p.sb + col) : 0.f, in && p.bias ? load_f32(p.bias + col) : 0.f};
}

// Scales W columns of a warp's 32 rows and writes them out through the warp's 2 KB of staging.  ok = false: NaN.
// TILES (rows that start and end on 16-byte boundaries): W columns are 64 bytes, copied as a box in the 64-byte swizzle (16-byte pieces by
// lane: no bank conflicts) that clips at the matrix and runs on while the next columns are scaled.  Else W = 16, two rows
// of 16 elements an access.  (32-byte stores by each lane into its own row cost a cache line an access: 3500 cycles for
// 32 x 32 fp32 against a stage's 513.)
template <typename T, int W, bool TILES>
__device__ __forceinline__ void finish_chunk(const Product8& p, const CUtensorMap* map_o, const uint32_t (&r)[W], bool ok, float sa, ColumnScale cs,
                                             uint32_t piece, uint64_t row0, uint64_t col, unsigned char* stage, uint32_t lane) {
    static_assert(TILES ? W * sizeof(T) == 64 : W == 16, "2 KB of staging");
    if (TILES) {
        if (lane == 0) tile_store_wait_read<0>();
        __syncwarp();
    }
    float* scales = reinterpret_cast<float*>(stage);
    if (W == 32 || (lane >> 4) == piece) {
        scales[lane & (W - 1)] = cs.sb;
        scales[W + (lane & (W - 1))] = cs.bias;
    }
    __syncwarp();
    float v[W];
#pragma unroll
    for (int j = 0; j < W; j += 4) {
        const float4 sb = *reinterpret_cast<const float4*>(scales + j);
        v[j] = __fmul_rn(__fmul_rn((float)(int)r[j], sa), sb.x);
        v[j + 1] = __fmul_rn(__fmul_rn((float)(int)r[j + 1], sa), sb.y);
        v[j + 2] = __fmul_rn(__fmul_rn((float)(int)r[j + 2], sa), sb.z);
        v[j + 3] = __fmul_rn(__fmul_rn((float)(int)r[j + 3], sa), sb.w);
    }
    if (p.bias) {
#pragma unroll
        for (int j = 0; j < W; j += 4) {
            const float4 bi = *reinterpret_cast<const float4*>(scales + W + j);
            v[j] = __fadd_rn(v[j], bi.x);
            v[j + 1] = __fadd_rn(v[j + 1], bi.y);
            v[j + 2] = __fadd_rn(v[j + 2], bi.z);
            v[j + 3] = __fadd_rn(v[j + 3], bi.w);
        }
    }
    if (!ok) {
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] = CUDART_NAN_F;
    }
    __syncwarp();
    if (row0 >= p.m || col >= p.n) return;
    if constexpr (TILES) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint4 w;
            if constexpr (W == 16) w = make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
            else w = make_uint4(pack2<T>(v[8 * i], v[8 * i + 1]), pack2<T>(v[8 * i + 2], v[8 * i + 3]), pack2<T>(v[8 * i + 4], v[8 * i + 5]), pack2<T>(v[8 * i + 6], v[8 * i + 7]));
            *reinterpret_cast<uint4*>(stage + lane * 64 + ((i ^ ((lane >> 1) & 3)) * 16)) = w;
        }
        smem_to_copies();
        __syncwarp();
        if (lane == 0) tile_store(map_o, (int32_t)col, (int32_t)row0, smem_u32(stage));
    } else {
        float* f = reinterpret_cast<float*>(stage);        // row i's column c at 16 i + (c ^ (i & 15))
#pragma unroll
        for (int j = 0; j < W; ++j) f[lane * 16 + (j ^ (lane & 15))] = v[j];
        __syncwarp();
        const uint32_t c = lane & 15, r1 = lane >> 4;
        const uint32_t n = p.m - row0 < 32 ? (uint32_t)(p.m - row0) : 32u;
        if (col + c < p.n) {
            T* out = static_cast<T*>(p.out) + (row0 + r1) * p.ldo + col + c;
            const uint64_t step = 2 * p.ldo;
            if (n == 32) {
#pragma unroll
                for (uint32_t i = 0; i < 32; i += 2, out += step) *out = from_f32<T>(f[(i + r1) * 16 + (c ^ ((i + r1) & 15))]);
            } else {
                for (uint32_t i = r1; i < n; i += 2, out += step) *out = from_f32<T>(f[i * 16 + (c ^ (i & 15))]);
            }
        }
        __syncwarp();
    }
}

// 64 columns of a warp's 32 rows from tensor memory, W at a time; `done` runs when the last have been read.
template <typename T, int W, bool TILES, class Done>
__device__ __forceinline__ void finish_columns(const Product8& p, const CUtensorMap* map_o, uint32_t tmem, bool ok, float sa, const ColumnScale (&cs)[2],
                                               uint64_t row0, uint64_t col, unsigned char* stage, uint32_t lane, Done&& done) {
#pragma unroll
    for (int i = 0; i < 64 / W; ++i) {
        uint32_t r[W];
        if (ok) {
            if constexpr (W == 32) tmem_ld32(tmem + i * W, r);
            else tmem_ld16(tmem + i * W, r);
            tmem_wait_ld();
        }
        if (i == 64 / W - 1) done();
        finish_chunk<T, W, TILES>(p, map_o, r, ok, sa, cs[i * W / 32], i & 1, row0, col + i * W, stage, lane);
    }
}

// T: element type of the (first) output; DUAL: the second one's is fp32.
template <typename T, bool SPLIT, bool TILES, bool DUAL>
__global__ void __launch_bounds__(kPairThreads, 1)
    product8_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_o,
                         const __grid_constant__ PairMaps maps2, const __grid_constant__ PairArgs args, uint32_t split) {
    static_assert(!(SPLIT && DUAL) && (TILES || !DUAL), "two products are whole tiles, by tiled copies");
    extern __shared__ unsigned char dyn[];
    __shared__ volatile uint32_t sh_tmem, sh_failed;
    const uint32_t data = (smem_u32(dyn) + 1023u) & ~1023u;
    unsigned char* stages = dyn + (data - smem_u32(dyn));
    const uint32_t bars = data + kPairStages * kPairStage + 16 * kStageStride;
    const auto full = [&](uint32_t s) { return bars + 16u * s; };
    const auto empty = [&](uint32_t s) { return bars + 16u * s + 8u; };
    const uint32_t acc_full = bars + 16u * kPairStages, acc_empty = acc_full + 16u, drain = acc_full + 32u, ready = acc_full + 40u;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, in_cluster = cluster_rank();
    const uint32_t rank = in_cluster & 1u, even = in_cluster & ~1u;            // the pair's CTA that issues
    const uint32_t part = SPLIT ? in_cluster >> 1 : 0, parts = SPLIT ? split : 1;
    const uint32_t pair = (blockIdx.x >> 1) / parts, pairs = (gridDim.x >> 1) / parts;
    TileWalk walk = {};
    walk.start<DUAL>(args, pair, pairs);
    const auto k_first = [&] { return SPLIT ? walk.job[0].kblocks * part / parts : 0u; };
    const auto k_last = [&] { return SPLIT ? walk.job[0].kblocks * (part + 1) / parts : walk.job[DUAL ? walk.cur : 0].kblocks; };

    if (threadIdx.x == 0) {
        sh_failed = 0;
        for (uint32_t s = 0; s < kPairStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (uint32_t i = 0; i < 2; ++i) {
            mbar_init(acc_full + 8 * i, 1);
            mbar_init(acc_empty + 8 * i, 32);              // sixteen warps of either CTA
        }
        mbar_init(drain, 1);
        mbar_init(ready, 1);
        mbar_init_fence();
        map_prefetch(&map_a);
        map_prefetch(&map_b);
    }
    cluster_sync_all();
    grid_wait();
    // Tensor memory is taken only now: a launch that held it while it waits could keep the one it waits for (which need not
    // be this library's) from ever getting its own.  The first copies travel meanwhile.
    if (warp == 17) {
        tmem_alloc<2>(smem_u32((const void*)&sh_tmem), 2 * kPairTile);
        if (rank == 1 && lane == 0) cluster_arrive(cluster_map(ready, even));
    }
    if (warp != 16) {
        umma_fence_before();
        asm volatile("bar.sync 1, 544;" ::: "memory");     // the seventeen warps that use it
        umma_fence_after();
        grid_go();
    }

    if (warp == 16 && lane == 0) {
        // ---- feed: this CTA's rows of either operand, completion counted on the even CTA's barrier
        uint32_t it = 0, s = 0, parity = 1;                // parity of the stage's last release (the first use waits for none)
        bool ok = true;
        while (ok && walk.step<DUAL>()) {
            const int32_t ya = (int32_t)(walk.tm * kPairTile + rank * 128), yb = (int32_t)(walk.tn * kPairTile + rank * 128);
            const CUtensorMap *from_a = DUAL && walk.cur ? &maps2.a : &map_a, *from_b = DUAL && walk.cur ? &maps2.b : &map_b;
            const int32_t x1 = (int32_t)(k_last() * 128);
            for (int32_t x = (int32_t)(k_first() * 128); x < x1; x += 128, ++it) {
                if (it >= kPairStages && !mbar_wait(empty(s), parity)) { ok = false; break; }
                if (rank == 0) mbar_expect_tx(full(s), 2 * kPairStage);
                const uint32_t dst = data + s * kPairStage, bar = cluster_map(full(s), even);
                tile_load<2>(dst, from_a, x, ya, bar);
                tile_load<2>(dst + kPairHalf, from_b, x, yb, bar);
                if (++s == kPairStages) { s = 0; parity ^= 1u; }
            }
        }
        if (!ok) {                                         // the odd CTA cannot see its copies land: leave them a millisecond
            sh_failed = 1;
            for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        }
        // no CTA of the pair may leave before its copies have landed and the last releases of its stages have arrived
        for (uint32_t j = it > kPairStages ? it - kPairStages : 0; j < it; ++j) {
            if (rank == 0) (void)mbar_wait(full(j % kPairStages), (j / kPairStages) & 1u);
            if (ok && !mbar_wait(empty(j % kPairStages), (j / kPairStages) & 1u)) ok = false;
        }
    } else if (warp == 17 && lane == 0 && rank == 0) {
        // ---- issue
        constexpr uint32_t idesc = umma_idesc_s8(256, kPairTile);
        const uint16_t both = (uint16_t)(3u << even);
        uint32_t s = 0, parity = 0, n_acc = 0;
        bool ok = mbar_wait(ready, 0);                     // the odd CTA has its tensor memory
        for (; ok && walk.step<DUAL>(); ++n_acc) {
            const uint32_t acc = n_acc & 1u, use = n_acc >> 1, blocks = k_last() - k_first(), into = sh_tmem + acc * kPairTile;
            // instructions of the last block: 32 codes each
            const uint32_t rest = (uint32_t)((args.p[DUAL ? walk.cur : 0].k + 31) / 32) - (k_last() - 1) * 4, last_steps = rest < 4 ? rest : 4;
            if (use > 0 && !mbar_wait(acc_empty + 8 * acc, (use - 1) & 1u)) { ok = false; break; }
            umma_fence_after();
            for (uint32_t kb = 0; kb < blocks; ++kb) {
                if (!mbar_wait(full(s), parity)) { ok = false; break; }
                umma_fence_after();
                const uint64_t da = umma_desc(data + s * kPairStage), db = umma_desc(data + s * kPairStage + kPairHalf);
                if (kb + 1 < blocks || last_steps == 4) {
                    umma_s8<2>(into, da, db, idesc, kb > 0);
                    umma_s8<2>(into, da + 2, db + 2, idesc, true);
                    umma_s8<2>(into, da + 4, db + 4, idesc, true);
                    umma_s8<2>(into, da + 6, db + 6, idesc, true);
                } else {
                    for (uint32_t j = 0; j < last_steps; ++j) umma_s8<2>(into, da + 2 * j, db + 2 * j, idesc, kb > 0 || j > 0);
                }
                umma_commit_pair(empty(s), both);
                if (++s == kPairStages) { s = 0; parity ^= 1u; }
            }
            if (ok) umma_commit_pair(acc_full + 8 * acc, both);
        }
        if (!ok) {
            sh_failed = 1;
            umma_commit_pair(drain, (uint16_t)(1u << even));
            (void)mbar_wait(drain, 0);
        }
        // the hand-backs that no further tile waits for come from the other CTA too: they arrive before this one may leave
        if (!SPLIT)
            for (uint32_t j = n_acc > 2 ? n_acc - 2 : 0; j < n_acc; ++j) (void)mbar_wait(acc_empty + 8 * (j & 1u), (j >> 1) & 1u);
    }
    __syncwarp();
    unsigned char* stage = stages + kPairStages * kPairStage + warp * kStageStride;
    const uint32_t quad = warp & 3, group = warp >> 2, row_in = rank * 128 + quad * 32;
    constexpr int kWidth = TILES && sizeof(T) == 2 ? 32 : 16;
    if constexpr (!SPLIT) {
        if (warp < 16) {
            // ---- write out: rows 32 quad + lane of this CTA's 128, 64 columns
            uint32_t n_acc = 0;
            bool ok = true;
            for (; walk.step<DUAL>(); ++n_acc) {
                const uint32_t acc = n_acc & 1u, use = n_acc >> 1;
                const Product8& p = args.p[DUAL ? walk.cur : 0];
                const uint64_t row0 = (uint64_t)walk.tm * kPairTile + row_in, col0 = (uint64_t)walk.tn * kPairTile + group * 64;
                const float sa = row0 + lane < p.m ? load_f32(p.sa + row0 + lane) : 0.f;
                const ColumnScale cs[2] = {column_scale(p, col0 + lane), column_scale(p, col0 + 32 + lane)};
                if (ok && !mbar_wait(acc_full + 8 * acc, use & 1u)) ok = false;
                ok = __all_sync(kFullMask, ok && !sh_failed);
                umma_fence_after();
                const uint32_t from = sh_tmem + ((quad * 32) << 16) + acc * kPairTile + group * 64;
                const auto done = [&] {
                    umma_fence_before();                   // everything read: the next tile may overwrite it
                    __syncwarp();
                    if (lane == 0 && ok) cluster_arrive(cluster_map(acc_empty + 8 * acc, even));   // (a failure hands nothing back)
                };
                if (DUAL && walk.cur) finish_columns<float, 16, true>(p, &maps2.o, from, ok, sa, cs, row0, col0, stage, lane, done);
                else finish_columns<T, kWidth, TILES>(p, &map_o, from, ok, sa, cs, row0, col0, stage, lane, done);
            }
            if (TILES && lane == 0) tile_store_wait_all();
        }
        __syncwarp();
        __syncthreads();
        cluster_meet_all();                                // the odd CTA's memory is read until the last instruction of the even one
    } else {
        // ---- one tile: leave the other pairs their columns in shared memory, then add up and write out one's own.  The
        // exchange runs at 18 bytes a cycle and CTA whether it is loads from the other CTAs' memories or bulk copies into them
        // (64 KB a CTA in two parts, 3500 cycles); as loads it overlaps with the first columns' output.
        const uint32_t cols = kPairTile / parts, mine = part * cols;
        int4* sums = reinterpret_cast<int4*>(stages);      // [four columns][row]: a warp's access is contiguous; every copy
        bool ok = true;                                    // has landed and every instruction has read its operands
        const Product8& p = args.p[0];
        (void)walk.step<DUAL>();
        const uint64_t row0 = (uint64_t)walk.tm * kPairTile + row_in, col0 = (uint64_t)walk.tn * kPairTile + mine + group * 32;
        const bool own = warp < 16 && group * 32 < cols && row0 < p.m && col0 < p.n;   // 32 columns a warp, of one's own, in the matrix
        float sa = 0.f;
        ColumnScale cs = {};
        if (warp < 16) {
            if (row0 + lane < p.m) sa = load_f32(p.sa + row0 + lane);
            if (own) cs = column_scale(p, col0 + lane);
            ok = mbar_wait(acc_full, 0);
            umma_fence_after();
            if (!ok) sh_failed = 1;
#pragma unroll 1
            for (uint32_t ch = 0; ch < 2; ++ch) {
                const uint32_t c = group * 64 + ch * 32;
                if (c >= mine && c < mine + cols) continue;
                uint32_t r[32];
                tmem_ld32(sh_tmem + ((quad * 32) << 16) + c, r);
                tmem_wait_ld();
                int4* to = sums + (c / 4) * 128 + quad * 32 + lane;
#pragma unroll
                for (int j = 0; j < 32; j += 4) to[j / 4 * 128] = make_int4((int)r[j], (int)r[j + 1], (int)r[j + 2], (int)r[j + 3]);
            }
            umma_fence_before();
        }
        cluster_sync_all();
        uint32_t r[32];
        if (own) {
            umma_fence_after();
            const uint32_t c = mine + group * 32;
            const auto fetch = [&](uint32_t q, int4 (&v)[8]) {
                const uint32_t from = cluster_map(data + ((c / 4) * 128 + quad * 32 + lane) * 16, ((part + q) & (parts - 1)) * 2 + rank);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = cluster_ld4(from + j * 2048);
            };
            int4 v[8];
            fetch(1, v);
            ok = cluster_all_zero(smem_u32((const void*)&sh_failed), 2 * parts);
            tmem_ld32(sh_tmem + ((quad * 32) << 16) + c, r);
            tmem_wait_ld();
#pragma unroll 1
            for (uint32_t q = 1; q < parts; ++q) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    r[4 * j] += (uint32_t)v[j].x;
                    r[4 * j + 1] += (uint32_t)v[j].y;
                    r[4 * j + 2] += (uint32_t)v[j].z;
                    r[4 * j + 3] += (uint32_t)v[j].w;
                }
                if (q + 1 < parts) fetch(q + 1, v);
            }
        }
        __syncwarp();
        cluster_arrive_all();                              // done with the others' sums
        if (own) {
            if constexpr (kWidth == 32) {
                finish_chunk<T, 32, TILES>(p, &map_o, r, ok, sa, cs, 0, row0, col0, stage, lane);
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t half[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) half[j] = r[16 * i + j];
                    finish_chunk<T, 16, TILES>(p, &map_o, half, ok, sa, cs, i, row0, col0 + 16 * i, stage, lane);
                }
            }
            if (TILES && lane == 0) tile_store_wait_all();
        }
        __syncwarp();
        cluster_wait_all();                                // nobody leaves while its sums are being read
    }
    if (warp == 17) tmem_free<2>(sh_tmem, 2 * kPairTile);
}

// ---- few rows: 128 x NT tiles, the contraction split over a cluster ------------------------------------
// The 128 rows are rows of b, the NT columns rows of a (tokens): with few tokens the weights are the long side, and an
// output row then runs along the lanes.  The CTAs of a cluster take consecutive parts of the contraction, leave
// their int32 sums in shared memory and each write out a part of the columns, summed over the cluster's shared
// memories.  Bound by the weights' traffic and 3.5 us of launch, set-up and last meeting: 9 x 16384 x 2048 10.4 us with the
// weights from memory (3.3 TB/s).  Warps: 0-3 write out, 4 feeds, 5 issues.
constexpr int kSlimThreads = 192;
// Rows of a that a tile holds at most; which products are taken: see takes_slim.
constexpr uint64_t kSlimRows = 64;
template <int NT> struct SlimGeom {
    static constexpr uint32_t kA = 128 * 128, kB = NT * 128, kStage = kA + kB;
    static constexpr uint32_t kStages = 4;
    static constexpr uint32_t kColumns = NT < 32 ? 32 : NT;
    static constexpr uint32_t kSmem = 1024 + kStages * kStage + 256;
    static_assert(kStages * kStage >= 128 * NT * 4, "the stages also hold the sums");
};

template <int NT, typename T>
__global__ void __launch_bounds__(kSlimThreads, 2)
    product8_slim_kernel(const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ Product8 p,
                         uint32_t split) {
    using G = SlimGeom<NT>;
    extern __shared__ unsigned char dyn[];
    __shared__ uint32_t sh_tmem;
    __shared__ float sh_sa[NT];
    __shared__ volatile uint32_t sh_failed;
    const uint32_t data = (smem_u32(dyn) + 1023u) & ~1023u;
    int4* sums = reinterpret_cast<int4*>(dyn + (data - smem_u32(dyn)));     // [four columns][row]: a warp's access is contiguous
    const uint32_t bars = data + G::kStages * G::kStage;
    const auto full = [&](uint32_t s) { return bars + 16u * s; };
    const auto empty = [&](uint32_t s) { return bars + 16u * s + 8u; };
    const uint32_t acc_full = bars + 16u * G::kStages, drain = acc_full + 8u;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t part = blockIdx.x % split, tn = blockIdx.x / split;
    const uint32_t kblocks = (uint32_t)((p.k + 127) / 128);
    const uint32_t kb0 = (uint32_t)((uint64_t)kblocks * part / split), kb1 = (uint32_t)((uint64_t)kblocks * (part + 1) / split);
    const uint32_t n = kb1 - kb0;

    if (threadIdx.x == 0) {
        sh_failed = 0;
        for (uint32_t s = 0; s < G::kStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        mbar_init(acc_full, 1);
        mbar_init(drain, 1);
        mbar_init_fence();
    }
    __syncthreads();
    grid_wait();
    if (warp == 5) tmem_alloc<1>(smem_u32(&sh_tmem), G::kColumns);         // only now: see the pair kernel
    if (warp != 4) {
        umma_fence_before();
        asm volatile("bar.sync 2, 160;" ::: "memory");
        umma_fence_after();
        grid_go();
    }
    const uint32_t tmem = sh_tmem;

    if (warp == 4 && lane == 0) {
        const int32_t yb = (int32_t)(tn * 128);
        uint32_t i = 0;
        for (; i < n; ++i) {
            const uint32_t s = i % G::kStages, use = i / G::kStages;
            if (use > 0 && !mbar_wait(empty(s), (use - 1) & 1u)) { sh_failed = 1; break; }
            mbar_expect_tx(full(s), G::kStage);
            const uint32_t dst = data + s * G::kStage;
            tile_load<1>(dst, &map_b, (int32_t)((kb0 + i) * 128), yb, full(s));
            tile_load<1>(dst + G::kA, &map_a, (int32_t)((kb0 + i) * 128), 0, full(s));
        }
        // every copy has landed and every release has arrived before the CTA may leave
        for (uint32_t j = i > G::kStages ? i - G::kStages : 0; j < i; ++j) {
            (void)mbar_wait(full(j % G::kStages), (j / G::kStages) & 1u);
            if (!sh_failed && !mbar_wait(empty(j % G::kStages), (j / G::kStages) & 1u)) sh_failed = 1;
        }
    } else if (warp == 5 && lane == 0) {
        constexpr uint32_t idesc = umma_idesc_s8(128, NT);
        bool ok = true;
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t s = i % G::kStages;
            if (!mbar_wait(full(s), (i / G::kStages) & 1u)) { ok = false; break; }
            umma_fence_after();
            const uint64_t db = umma_desc(data + s * G::kStage), da = umma_desc(data + s * G::kStage + G::kA);
            const uint64_t left = p.k - (uint64_t)(kb0 + i) * 128;
            const uint32_t steps = left >= 128 ? 4u : (uint32_t)((left + 31) / 32);
            for (uint32_t j = 0; j < steps; ++j) umma_s8<1>(tmem, db + 2 * j, da + 2 * j, idesc, i > 0 || j > 0);
            umma_commit(empty(s));
        }
        if (!ok) {
            sh_failed = 1;
            __threadfence_block();
        }
        umma_commit(acc_full);
        if (!ok) {
            umma_commit(drain);
            (void)mbar_wait(drain, 0);
        }
    }
    __syncwarp();

    bool ok = true;
    const uint64_t chan = (uint64_t)tn * 128 + warp * 32 + lane;
    float sb = 0.f, bias = 0.f;
    if (warp < 4) {                                        // scales ahead of the sums: a load between two stores costs its whole latency
        if (threadIdx.x < NT) sh_sa[threadIdx.x] = threadIdx.x < p.m ? load_f32(p.sa + threadIdx.x) : 0.f;
        if (chan < p.n) {
            sb = load_f32(p.sb + chan);
            if (p.bias) bias = load_f32(p.bias + chan);
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
        ok = mbar_wait(acc_full, 0);
        umma_fence_after();
    }
    T* out = static_cast<T*>(p.out);
    const auto put = [&](uint32_t c, int acc, bool good) {
        if (chan < p.n && c < p.m)
            out[c * p.ldo + chan] = from_f32<T>(good ? scaled(acc, sh_sa[c], sb, p.bias, bias) : CUDART_NAN_F);
    };
    if (split == 1) {
        if (warp < 4) {
            const bool good = __all_sync(kFullMask, ok && !sh_failed);
#pragma unroll 1
            for (uint32_t c = 0; c < NT; c += 16) {
                uint32_t r[16];
                if (c >= p.m) break;
                tmem_ld16(tmem + ((warp * 32) << 16) + c, r);
                tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; ++j) put(c + j, (int)r[j], good);
            }
        }
        umma_fence_before();
        __syncthreads();
    } else {
        if (warp < 4) {
            if (!ok) sh_failed = 1;
#pragma unroll 1
            for (uint32_t c = 0; c < NT; c += 16) {
                uint32_t r[16];
                tmem_ld16(tmem + ((warp * 32) << 16) + c, r);
                tmem_wait_ld();
                int4* to = sums + (c / 4) * 128 + warp * 32 + lane;
#pragma unroll
                for (int j = 0; j < 16; j += 4) to[j / 4 * 128] = n > 0 ? make_int4((int)r[j], (int)r[j + 1], (int)r[j + 2], (int)r[j + 3]) : make_int4(0, 0, 0, 0);
            }
        }
        umma_fence_before();
        cluster_sync_all();                                // every part's sums are in place
        constexpr uint32_t kMost = NT / 2;                 // columns of a part, of two at least
        const uint32_t cols = NT / split < 4 ? 4 : NT / split, c0 = cols * part;
        const uint32_t end = c0 >= p.m ? 0 : p.m - c0 < cols ? (uint32_t)p.m - c0 : cols;
        const bool mine = warp < 4 && (uint64_t)tn * 128 + warp * 32 < p.n;
        int4 a[kMost / 4];
        bool good = false;
        if (mine) {
            good = cluster_all_zero(smem_u32((const void*)&sh_failed), split);
            const uint32_t at = data + (c0 / 4 * 128 + warp * 32 + lane) * 16;
#pragma unroll
            for (uint32_t i = 0; i < kMost / 4; ++i) {
                if (4 * i >= end) break;
                int4 v[8];
#pragma unroll
                for (uint32_t q = 0; q < 8; ++q) v[q] = q < split ? cluster_ld4(cluster_map(at + i * 2048, q)) : make_int4(0, 0, 0, 0);
                a[i] = v[0];
#pragma unroll
                for (int q = 1; q < 8; ++q) {
                    a[i].x += v[q].x;
                    a[i].y += v[q].y;
                    a[i].z += v[q].z;
                    a[i].w += v[q].w;
                }
            }
        }
        __syncwarp();
        cluster_arrive_all();                              // done with the others' sums
        if (mine) {
#pragma unroll
            for (uint32_t i = 0; i < kMost / 4; ++i) {
                if (4 * i >= end) break;
                put(c0 + 4 * i, a[i].x, good);
                put(c0 + 4 * i + 1, a[i].y, good);
                put(c0 + 4 * i + 2, a[i].z, good);
                put(c0 + 4 * i + 3, a[i].w, good);
            }
        }
        __syncwarp();
        cluster_wait_all();                                // nobody leaves while its sums are being read
    }
    if (warp == 5) tmem_free<1>(tmem, G::kColumns);
}

// ---- host ------------------------------------------------------------------------------------------
// `lines` lines of k codes, boxes of 128 codes x `box` lines; codes beyond a line's end read as zero.
bool make_map(CUtensorMap* map, const int8_t* codes, uint64_t lines, uint64_t k, uint64_t ld, uint32_t box) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {k, lines}, strides[1] = {ld};
    const cuuint32_t boxes[2] = {128, box}, steps[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(codes), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Boxes of 64 bytes x 32 rows of the output.
bool make_out_map(CUtensorMap* map, const Product8& p, uint32_t element) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {p.n, p.m}, strides[1] = {p.ldo * element};
    const cuuint32_t boxes[2] = {64 / element, 32}, steps[2] = {1, 1};
    return encode(map, element == 4 ? CU_TENSOR_MAP_DATA_TYPE_UINT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, p.out, dims, strides, boxes, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The dynamic shared-memory opt-in of one kernel instantiation, once per device.
template <typename K> cudaError_t allow_smem(K kernel, uint32_t bytes, PerDevice<bool>& done) {
    const int slot = device_slot();
    if (slot >= 0 && done.v[slot]) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess && slot >= 0) done.v[slot] = true;
    return e;
}

template <typename T, bool SPLIT, bool TILES, bool DUAL>
cudaError_t launch_pair_as(const Product8& p, const Product8* p2, uint32_t split, cudaStream_t st) {
    static PerDevice<bool> done;
    const auto kernel = product8_pair_kernel<T, SPLIT, TILES, DUAL>;
    cudaError_t e = allow_smem(kernel, kPairSmem, done);
    if (e != cudaSuccess) return e;
    PairArgs args = {};
    PairMaps maps[2] = {};
    uint64_t tiles = 0;
    for (int i = 0; i < (DUAL ? 2 : 1); ++i) {
        const Product8& q = args.p[i] = i ? *p2 : p;
        if (!make_map(&maps[i].a, q.a, q.m, q.k, q.lda, 128) || !make_map(&maps[i].b, q.b, q.n, q.k, q.ldb, 128)) return cudaErrorNotSupported;
        if (TILES && !make_out_map(&maps[i].o, q, i ? 4 : sizeof(T))) return cudaErrorNotSupported;
        tiles += (q.m + 255) / 256 * ((q.n + 255) / 256);
    }
    const uint64_t pairs = (uint64_t)sm_count_now() / 2;
    if (tiles >= (1ull << 31)) return cudaErrorInvalidValue;
    return launch_layer(kernel, (unsigned)(2 * (SPLIT ? tiles * split : tiles < pairs ? tiles : pairs)), kPairThreads, kPairSmem, 2 * split, st,
                        maps[0].a, maps[0].b, maps[0].o, maps[1], args, split);
}
// Whether the output may leave by tiled copies.  Its rows start on 16-byte boundaries, as the copies need, and end on one: a copy
// clips at the matrix in pieces of 16 bytes and would clear up to 15 bytes after a row that ends inside one.
bool rows_by_tiles(const Product8& p) {
    const uint64_t e = type_bytes(p.type);
    return (reinterpret_cast<uintptr_t>(p.out) | p.ldo * e | p.n * e) % 16 == 0;
}
template <typename T> cudaError_t launch_pair(const Product8& p, uint32_t split, cudaStream_t st) {
    const bool tiles = rows_by_tiles(p);
    if (split > 1) return tiles ? launch_pair_as<T, true, true, false>(p, nullptr, split, st) : launch_pair_as<T, true, false, false>(p, nullptr, split, st);
    return tiles ? launch_pair_as<T, false, true, false>(p, nullptr, 1, st) : launch_pair_as<T, false, false, false>(p, nullptr, 1, st);
}

// Clusters of `split` pairs that run at once on this device.
template <typename T> uint64_t resident_clusters(uint32_t split) {
    static PerDevice<int> known[2];
    const int slot = device_slot();
    PerDevice<int>& table = known[split == 2 ? 0 : 1];
    if (slot >= 0 && table.v[slot] > 0) return (uint64_t)table.v[slot] - 1;
    static PerDevice<bool> done;
    const auto kernel = product8_pair_kernel<T, true, true, false>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * split);
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = kPairSmem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2 * split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (allow_smem(kernel, kPairSmem, done) != cudaSuccess || cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
        (void)cudaGetLastError();
        n = 0;
    }
    if (slot >= 0) table.v[slot] = n + 1;
    return (uint64_t)n;
}

// Tiles that leave pairs idle: split the contraction, four stages of it at least to a part, as long as all clusters run
// at once (512 x 4096 x 4096, 32 tiles: 13.2 us whole, 12.0 in two parts, 29.5 in four, where clusters of eight queue; 200 x
// 4096 x 4096, 16 tiles: 13.1, 11.0, 19.1).
template <typename T> uint32_t pair_split(const Product8& p) {
    const uint64_t tiles = (p.m + 255) / 256 * ((p.n + 255) / 256), kblocks = (p.k + 127) / 128;
    uint32_t split = 1;
    while (split < 4 && kblocks >= split * 8 && tiles <= resident_clusters<T>(split * 2)) split *= 2;
    return split;
}

// Which kernel a product of few rows takes.  The slim kernel's time grows with the rows (2 to 3 us from 24 to 64: more output by
// scalar stores), the pairs' does not: above 32 rows the pairs win where their tiles, whole or in two parts, fill half a wave
// or more and not more than one.  Slim and pairs, us, weights from memory:
//   24 rows: 16384 x 2048 11.1, 11.3   8192 x 4096 12.1, 14.2   12288 x 4096 16.2, 18.5   5120 x 1024 6.7, 6.5
//   48 rows: 16384 x 2048 12.4, 11.1   8192 x 4096 13.9, 12.1   12288 x 4096 17.5, 14.5   5120 x 1024 8.5, 7.1
//   64 rows, less than half a wave: 1024 x 1024 5.3, 6.2   4096 x 4096 9.1, 10.4   4608 x 8192 13.6, 15.4
//   64 rows, four parts: 2560 x 2560 7.4, 7.7   more than a wave: 28672 x 4096 26.0, 26.8   28672 x 8192 46.6, 52.4
//   (but 65536 x 1024 22.9, 19.0)
template <typename T> bool takes_slim(const Product8& p) {
    if (p.m > kSlimRows || p.m <= 32) return p.m <= 32;
    const uint64_t split = pair_split<T>(p), units = (p.n + 255) / 256 * split, pairs = (uint64_t)sm_count_now() / 2;
    return split > 2 || 2 * units < pairs || units > pairs;
}

template <int NT, typename T> cudaError_t launch_slim(const Product8& p, uint32_t split, cudaStream_t st) {
    using G = SlimGeom<NT>;
    static PerDevice<bool> done;
    const auto kernel = product8_slim_kernel<NT, T>;
    cudaError_t e = allow_smem(kernel, G::kSmem, done);
    if (e != cudaSuccess) return e;
    CUtensorMap ma, mb;
    if (!make_map(&mb, p.b, p.n, p.k, p.ldb, 128) || !make_map(&ma, p.a, p.m, p.k, p.lda, NT)) return cudaErrorNotSupported;
    const uint64_t ctas = (p.n + 127) / 128 * split;
    if (ctas >= (1ull << 31)) return cudaErrorInvalidValue;
    return launch_layer(kernel, (unsigned)ctas, kSlimThreads, G::kSmem, split, st, mb, ma, p, split);
}

}  // namespace

bool product8_codes_tokens(uint64_t tokens, uint64_t k) { return tokens <= kStreamTokens && k <= 8ull * kStreamHold * stream_share(tokens); }

cudaError_t launch_linear8_stream(const void* x, uint64_t ldx, const Product8& p, cudaStream_t st) {
    return with_type(p.type, [&](auto t) {
        using T = decltype(t);
        const uint64_t kparts = (p.k + 255) / 256, ks = kparts >= 5 ? 8 : kparts >= 3 ? 4 : kparts;
        const uint64_t rounds = ((p.n + 15) / 16 * ks + 7) / 8, most = 2ull * sm_count_now();
        return launch_layer(product8_stream_kernel<T>, (unsigned)(rounds < most ? rounds : most), kStreamThreads, p.m * stream_pitch(p.k), 1, st,
                            static_cast<const T*>(x), ldx, p);
    });
}

cudaError_t launch_product8(const Product8& p, cudaStream_t st) {
    const uint64_t sms = (uint64_t)sm_count_now(), kblocks = (p.k + 127) / 128;
    return with_type(p.type, [&](auto t) {
        using T = decltype(t);
        if (takes_slim<T>(p)) {
            const uint64_t nt = p.m <= 16 ? 16 : p.m <= 32 ? 32 : 64;
            const uint64_t tiles = (p.n + 127) / 128;
            uint32_t split = 1;
            while (split < 8 && tiles * split * 2 <= sms && kblocks >= split * 4) split *= 2;
            if (nt == 16) return launch_slim<16, T>(p, split, st);
            if (nt == 32) return launch_slim<32, T>(p, split, st);
            return launch_slim<64, T>(p, split, st);
        }
        const uint32_t split = pair_split<T>(p);
        return launch_pair<T>(p, split, st);
    });
}

cudaError_t launch_product8_two(const Product8& p, const Product8& fp32, cudaStream_t st) {
    return with_type(p.type, [&](auto t) {
        using T = decltype(t);
        // one launch where each would be whole tiles anyway
        if (p.m > kSlimRows && fp32.m > kSlimRows && rows_by_tiles(p) && rows_by_tiles(fp32) && pair_split<T>(p) == 1 && pair_split<float>(fp32) == 1)
            return launch_pair_as<T, false, true, true>(p, &fp32, 1, st);
        const cudaError_t e = launch_product8(p, st);
        return e != cudaSuccess ? e : launch_product8(fp32, st);
    });
}

}  // namespace tng

using namespace tng;

extern "C" tng_status tng_product8(const int8_t* a_dev, uint64_t lda, const float* sa_dev, const int8_t* b_dev, uint64_t ldb,
                                   const float* sb_dev, const float* bias_dev, uint64_t m, uint64_t n, uint64_t k, void* out_dev,
                                   tng_dtype type, uint64_t ldo, void* stream) {
    if (!type_ok(type) || n < 1 || k < 1 || k > TNG_MAX_CONTRACTION || !dims_ok(m, n)) return TNG_ERR_INVALID_ARG;
    if (m == 0) return TNG_OK;
    if (!codes_ok(a_dev, k, lda) || !codes_ok(b_dev, k, ldb) || !sa_dev || !sb_dev || !aligned(sa_dev, 4) || !aligned(sb_dev, 4) ||
        !aligned(bias_dev, 4) || !matrix_ok(out_dev, type, n, ldo))
        return TNG_ERR_INVALID_ARG;
    const Product8 p{a_dev, b_dev, lda, ldb, sa_dev, sb_dev, bias_dev, m, n, k, out_dev, type, ldo};
    return layer_status(launch_product8(p, static_cast<cudaStream_t>(stream)));
}
