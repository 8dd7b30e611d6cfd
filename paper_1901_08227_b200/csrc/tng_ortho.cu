// Orthogonalised updates: X = V / |V| (Frobenius), then X <- (a I + b G + c G^2) X with G = X X^T, a few times over.  Every step is an
// odd polynomial of the singular values alone, so that they move towards one while the singular vectors stay.
//
// A step is three products: G = X X^T and B = a I + b G + c G G (both symmetric: only the tiles on and below the diagonal are
// computed, and written twice), then B X.  With s the shorter side and l the longer, 3 s^2 l + s^3 operations.
//
// Accuracy.  Every factor is held as two fp16 numbers, hi + lo, 22 bits together, times a power of two that keeps the bounds below in
// fp16's range; a product is three (hi lo, lo hi, hi hi), lo lo being below 2^-22 of it.  The scales are fixed, so that the smallest steps are 2^-38 of
// |V| for X, 2^-37 and 2^-36 for G and B: 22 bits hold for entries of X from 2^-16 of |V| up, and a row or column far smaller than the
// rest keeps fewer (256 x 512, five steps, 32 rows at 1e-4 of the others: off by 3.8e-6 of their norm, at 1e-6 3.7e-4, at 1e-8 3.7e-2; fp32
// products 5.3e-7 throughout).  The error of the whole is below that of fp32 products (512 x 512: 1.5e-6 and 2.1e-6 of the norm).
// (bf16 factors alone, 8 bits, would do for the singular values that are near one, but a step multiplies what lies in the
// directions of the small ones by up to a: after five steps rounding noise of 2^-9 has grown by a factor of hundreds there.)  The tensor
// memory's sums lose about half a step of fp32 with every instruction, all in one direction; so they run over one or two
// blocks of the contraction only, and the chunks are added to nearest in registers.
//
// Long matrices with 16-bit results take several steps (up to kMostGroup) with one look at X: G after a step is B G B, so that only
// products of the shorter side's size lie between G = X X^T and the product of the Bs, which X then takes at once: for m steps
// 3 s^2 l + (4 m - 3) s^3 operations instead of 3 m s^2 l + m s^3 (4096 x 16384, five steps: 11.4 ms, so 6.3).  The rounding of B G B is
// several times that of X X^T and takes the result's error before its rounding from 1.5e-6 to 1.1e-5 of its entries (1024 x 4096: from 1.9e-6 to
// 6.0e-6): nothing beside bf16's 1.7e-3 or fp16's 2e-4, but more than fp32 products throughout leave (2.8e-6), so results in fp32 go step by
// step.
//
// Bounds (checked on the host for the given coefficients): singular values of X at most 2, so entries of X at most 2, of G 4, and of B
// 15; stored as X 2^14, G 2^13, B 2^12.
#include <math_constants.h>

#include <cmath>
#include <type_traits>

#include "tng_layers.cuh"
#include "tng_umma.cuh"

namespace tng {
namespace {

constexpr float kScaleX = 0x1p14f, kScaleG = 0x1p13f, kScaleB = 0x1p12f;
constexpr double kMostX = 2.0, kMostB = 15.0;
constexpr uint32_t kMostGroup = 3;

// A matrix held in two halves: `batch` of them, rows rounded up to 128, row stride ld.
struct Halves {
    __half *hi, *lo;
    uint64_t rows, cols, pad_rows, ld;
};

// ---- |V| and its two halves --------------------------------------------------------------------------------
// The sum of squares in 64 bits (no overflow, no underflow, and its rounding does not show), each block's share on its own.
constexpr uint32_t kNormBlocks = 128;
constexpr int kNormThreads = 512;
template <typename T>
__global__ void __launch_bounds__(kNormThreads) ortho_norm_kernel(const T* v, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t stride, double* part) {
    __shared__ double sh[kNormThreads / 32];
    grid_wait();
    grid_go();
    v += blockIdx.y * stride;
    double s = 0.0;
    constexpr int kAhead = 8;
    // a warp has a row at a time, eight loads a lane under way
    for (uint64_t r = (uint64_t)(threadIdx.x >> 5) * gridDim.x + blockIdx.x; r < rows; r += (uint64_t)(kNormThreads / 32) * gridDim.x) {
        const T* row = v + r * ld;
        for (uint64_t c = threadIdx.x & 31; c < cols; c += 32 * kAhead) {
            float e[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) e[i] = c + 32 * i < cols ? to_f32(row[c + 32 * i]) : 0.f;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) s += (double)e[i] * (double)e[i];
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(kFullMask, s, d);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kNormThreads / 32; ++i) s += sh[i];
        part[blockIdx.y * kNormBlocks + blockIdx.x] = s;
    }
}

__device__ __forceinline__ void split(float v, __half& hi, __half& lo) {
    hi = __float2half_rn(v);
    lo = __float2half_rn(__fsub_rn(v, __half2float(hi)));
}

// V / |V| in two halves, as it lies and transposed.  A block has 64 x 64 elements; they leave in pairs (rows are padded to 64).  The blocks of the
// longer side are counted by the grid's x: its y ends at 65535.
template <typename T>
__global__ void __launch_bounds__(256) ortho_split_kernel(const T* v, uint64_t ld, uint64_t stride, const double* part, const __grid_constant__ Halves as,
                                                          const __grid_constant__ Halves turned) {
    __shared__ __half hi[64][66], lo[64][66];
    __shared__ double total[4];
    grid_wait();
    grid_go();
    const uint32_t b = blockIdx.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool tall = as.rows > as.cols;
    const uint64_t r0 = (uint64_t)(tall ? blockIdx.x : blockIdx.y) * 64, c0 = (uint64_t)(tall ? blockIdx.y : blockIdx.x) * 64;
    v += b * stride;
    float e[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const uint64_t r = r0 + (threadIdx.x >> 6) + 4 * k, c = c0 + (threadIdx.x & 63);
        e[k] = r < as.rows && c < as.cols ? to_f32(v[r * ld + c]) : 0.f;
    }
    static_assert(kNormBlocks == 128, "four warps add up the shares");
    double s = threadIdx.x < kNormBlocks ? part[b * kNormBlocks + threadIdx.x] : 0.0;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(kFullMask, s, d);
    if (lane == 0 && warp < 4) total[warp] = s;
    __syncthreads();
    const double norm = sqrt((total[0] + total[1]) + (total[2] + total[3]));
    // (a norm that is not finite makes all of the matrix NaN, a zero one leaves it zero)
    const double f = norm == 0.0 ? 0.0 : norm < (double)CUDART_INF ? (double)kScaleX / norm : (double)CUDART_NAN_F;
#pragma unroll
    for (int k = 0; k < 16; ++k) split((float)((double)e[k] * f), hi[(threadIdx.x >> 6) + 4 * k][threadIdx.x & 63], lo[(threadIdx.x >> 6) + 4 * k][threadIdx.x & 63]);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t p = (threadIdx.x >> 5) + 8 * k, q = 2 * lane;
        if (r0 + p < as.rows && c0 + q < as.cols) {
            const uint64_t at = (b * as.pad_rows + r0 + p) * as.ld + c0 + q;
            *reinterpret_cast<__half2*>(as.hi + at) = __halves2half2(hi[p][q], hi[p][q + 1]);
            *reinterpret_cast<__half2*>(as.lo + at) = __halves2half2(lo[p][q], lo[p][q + 1]);
        }
        if (c0 + p < turned.rows && r0 + q < turned.cols) {
            const uint64_t at = (b * turned.pad_rows + c0 + p) * turned.ld + r0 + q;
            *reinterpret_cast<__half2*>(turned.hi + at) = __halves2half2(hi[q][p], hi[q + 1][p]);
            *reinterpret_cast<__half2*>(turned.lo + at) = __halves2half2(lo[q][p], lo[q + 1][p]);
        }
    }
}

// ---- products --------------------------------------------------------------------------------------------
// D = P Q^T of two matrices in halves, contraction along the rows of both, by pairs of CTAs on two SMs: tiles of 256 x 256 or 256 x 128
// outputs.  A CTA copies 128 rows of P and half the tile's rows of Q, both halves of them, for a stage of 64 of the contraction (12
// instructions).  The matrix unit would take 1536 cycles a stage for 256 x 256 and 768 for 256 x 128; measured 2000 (the sums' way into
// registers: two of them have all of the tensor memory) and 1150 (issue), so the narrow tiles are for matrices of few tiles.  (128 x 128
// tiles of one SM: 1580 cycles; they want 213 bytes a cycle of shared memory.)
// SPLIT (256 x 128): a cluster of 2 or 4 pairs takes consecutive parts of one tile's contraction; each then adds the others' sums, read
// from their shared memories, to its own for its share of the columns and writes those out.
// Warps: 0-15 add up and write out (a quarter of the rows and of the columns each), 16 feeds, 17 issues.  256 x 128: 17 and 18 issue
// every other sum each: an instruction takes its thread 54 cycles, a block with its waits and commits 1285, the matrix unit 768.
enum Kind { kGram = 0, kPoly = 1, kApply = 2, kLast = 3 };
constexpr int kThreads = 608;
constexpr uint32_t kBox = 128 * 128, kBlock = 64;
// (Stages of 32, twice as many, whose rows are 64 bytes: 2048 x 2048 x 8192 134 us instead of 113.)
// Staging of the output: buffers of 2 KB, two a warp where at most eight warps write (SPLIT).
template <uint32_t COLS, bool SPLIT> struct Geom {
    static constexpr uint32_t kQ = COLS / 2 * 128, kStage = 2 * kBox + 2 * kQ, kStages = COLS == 256 ? 3 : 4;
    static constexpr uint32_t kBuffers = SPLIT ? 2 : 1, kStaging = 2048 * kBuffers;
    static constexpr uint32_t kSmem = 1024 + kStages * kStage + (SPLIT ? 8 : 16) * kStaging + 256;
    // Blocks whose sum the tensor memory forms, and such sums under way: all of it.
    static constexpr uint32_t kChunk = COLS == 256 ? 2 : 1, kSums = 512 / COLS;
    static_assert(kSmem <= 227 * 1024, "shared memory of a CTA");
    static_assert(16 * kStages + 16 * kSums + 24 <= 256, "barriers");
    // A barrier's parity tells a phase only from its neighbours: a warp that waits for one phase has to have seen the one before.  So with two
    // issuing warps every stage and every place of a sum belongs to one of them.
    static constexpr uint32_t kIssuers = COLS == 128 ? 2 : 1;
    static_assert(kIssuers == 1 || (kChunk == 1 && kStages % kIssuers == 0 && kSums % kIssuers == 0), "a stage is waited for by one warp alone");
};
static_assert(128 * 128 * 4 <= Geom<128, true>::kStages * Geom<128, true>::kStage, "the stages also hold the sums");

struct OrthoMaps {
    CUtensorMap p[2], q[2], d[2], t[2];   // hi and lo of the factors, of D and (split products) of its transpose
};
struct OrthoArgs {
    uint64_t rows, cols, k;         // of D, and the contraction
    uint64_t pad_p, pad_q, pad_d;   // rows from one matrix of the batch to the next
    uint32_t batch, symmetric, split;
    float scale, linear, diagonal;  // D = scale * sum (+ linear * g + diagonal on the diagonal: kPoly)
    Halves g, t;                    // kPoly: the factor itself; D's transpose (D, if it is symmetric)
    void* out;                      // kLast
    uint64_t ldo, stride;
};

// A launch's tiles, 256 rows by `width` columns: by matrix, then by rows of tiles.  Symmetric products: those that reach below the
// diagonal; a block of 256 on it is computed whole, what lies left of it is written twice.
struct Tiles {
    uint32_t down, across, ratio, per, count, symmetric;
    __device__ __forceinline__ Tiles(const OrthoArgs& a, uint32_t width) {
        down = (uint32_t)((a.rows + 255) / 256);
        across = (uint32_t)((a.cols + width - 1) / width);
        ratio = 256 / width;
        symmetric = a.symmetric;
        per = symmetric ? ratio * (down * (down + 1) / 2) - (down * ratio - across) : down * across;
        count = per * a.batch;
    }
    __device__ __forceinline__ void at(uint32_t t, uint32_t& b, uint32_t& tm, uint32_t& tn) const {
        b = t / per;
        t -= b * per;
        if (symmetric) {
            const uint32_t u = t / ratio;
            tm = (uint32_t)((sqrtf(8.f * (float)u + 1.f) - 1.f) * 0.5f);
            while (tm * (tm + 1) / 2 > u) --tm;
            while ((tm + 1) * (tm + 2) / 2 <= u) ++tm;
            tn = t - ratio * (tm * (tm + 1) / 2);
        } else {
            // groups of eight rows of tiles, columns outside: neighbours in time share factors
            const uint32_t band = 8 * across, g = t / band, top = g * 8, high = down - top < 8 ? down - top : 8, r = t - g * band;
            tn = r / high;
            tm = top + (r - tn * high);
        }
    }
};

// 32 columns of a warp's 32 rows (lane = row) through 2 KB of staging by a tiled copy that clips at the matrix: the high halves of
// the values, or the low ones.  An element is kept as both halves in one register (high half in the high bits).
__device__ __forceinline__ float both_halves(float v) {
    __half hi, lo;
    split(v, hi, lo);
    return __uint_as_float((uint32_t)__half_as_ushort(hi) << 16 | __half_as_ushort(lo));
}
template <bool LO, uint32_t C, int BUFFERS, uint32_t N>
__device__ __forceinline__ void put_rows(const CUtensorMap* map, const float (&v)[N], int32_t x, int32_t y, unsigned char* stage, uint32_t lane) {
    if (lane == 0) tile_store_wait_read<BUFFERS - 1>();
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = __byte_perm(__float_as_uint(v[C + 8 * i + 2 * j]), __float_as_uint(v[C + 8 * i + 2 * j + 1]), LO ? 0x5410 : 0x7632);
        *reinterpret_cast<uint4*>(stage + lane * 64 + ((i ^ ((lane >> 1) & 3)) * 16)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    smem_to_copies();
    __syncwarp();
    if (lane == 0) tile_store(map, x, y, smem_u32(stage));
}
// The same transposed: row j of the box is column j, its 32 values the lanes'.
template <bool LO, uint32_t C, int BUFFERS, uint32_t N>
__device__ __forceinline__ void put_turned_staged(const CUtensorMap* map, const float (&v)[N], int32_t x, int32_t y, unsigned char* stage, uint32_t lane) {
    if (lane == 0) tile_store_wait_read<BUFFERS - 1>();
    __syncwarp();
#pragma unroll
    for (uint32_t j = 0; j < 32; ++j) {
        const uint32_t w = __float_as_uint(v[C + j]);
        *reinterpret_cast<uint16_t*>(stage + j * 64 + (((lane >> 3) ^ ((j >> 1) & 3)) * 16) + (lane & 7) * 2) = (uint16_t)(LO ? w : w >> 16);
    }
    smem_to_copies();
    __syncwarp();
    if (lane == 0) tile_store(map, x, y, smem_u32(stage));
}
// The same, both halves, straight into memory: neighbouring lanes exchange a value, so that each stores two of one column, and 16
// lanes 64 bytes.  Where staging is short (one buffer a warp) this is faster than copies (2048 x 8192 x 2048 186 -> 180 us), with more it
// is slower (512 x 512, five steps: 146 -> 157 us).
template <uint32_t C, uint32_t N>
__device__ __forceinline__ void put_turned(const Halves& t, const float (&v)[N], uint32_t b, uint64_t row0, uint64_t col, uint64_t rows, uint64_t cols, uint32_t lane) {
    const uint32_t odd = lane & 1;
    const uint64_t row = row0 + (lane & 30u);              // (a pair may end one past the last row: rows of t are padded to 64)
    uint64_t at = (b * t.pad_rows + col + odd) * t.ld + row;
#pragma unroll
    for (uint32_t j = 0; j < 32; j += 2, at += 2 * t.ld) {
        const uint32_t v0 = __float_as_uint(v[C + j]), v1 = __float_as_uint(v[C + j + 1]);
        const uint32_t got = __shfl_xor_sync(kFullMask, odd ? v0 : v1, 1);
        const uint32_t low = odd ? got : v0, high = odd ? v1 : got;        // rows `row` and `row` + 1 of column j + odd
        if (row < rows && col + j + odd < cols) {
            *reinterpret_cast<uint32_t*>(t.hi + at) = __byte_perm(low, high, 0x7632);
            *reinterpret_cast<uint32_t*>(t.lo + at) = __byte_perm(low, high, 0x5410);
        }
    }
}

// A warp's 32 columns from C of its sums, finished and written: see ortho_product_kernel.
template <int KIND, typename T, uint32_t C, int BUFFERS, uint32_t N>
__device__ __forceinline__ void finish(const OrthoMaps& maps, const OrthoArgs& a, float (&sum)[N], uint32_t b, uint64_t row0, uint64_t col, bool mirrored,
                                       unsigned char* stage, uint32_t lane) {
    if (col >= a.cols) return;
    if constexpr (KIND == kLast) {
        // two rows of 16 elements an access
        float* f = reinterpret_cast<float*>(stage);                        // row i's column j at 16 i + (j ^ (i & 15))
        T* out = static_cast<T*>(a.out) + b * a.stride;
        const uint32_t n = a.rows - row0 < 32 ? (uint32_t)(a.rows - row0) : 32u, j = lane & 15;
#pragma unroll
        for (uint32_t half = 0; half < 32; half += 16) {
            __syncwarp();
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) f[lane * 16 + (i ^ (lane & 15))] = __fmul_rn(sum[C + half + i], a.scale);
            __syncwarp();
            if (col + half + j < a.cols)
                for (uint32_t i = lane >> 4; i < n; i += 2) out[(row0 + i) * a.ldo + col + half + j] = from_f32<T>(f[i * 16 + (j ^ (i & 15))]);
        }
    } else {
        if constexpr (KIND == kPoly) {
            const uint64_t at = (b * a.g.pad_rows + row0 + lane) * a.g.ld + col;
#pragma unroll
            for (uint32_t i = 0; i < 32; i += 8) {         // (loads ahead of the sums: no faster, and more spills)
                const bool in = row0 + lane < a.rows && col + i < a.cols;
                const uint4 zero = make_uint4(0u, 0u, 0u, 0u), h = in ? load16(a.g.hi + at + i) : zero, l = in ? load16(a.g.lo + at + i) : zero;
                const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) {
                    const float2 x = unpack2<__half>(hw[j / 2]), y = unpack2<__half>(lw[j / 2]);
                    const float g = j & 1 ? x.y + y.y : x.x + y.x, d = row0 + lane == col + i + j ? a.diagonal : 0.f;
                    sum[C + i + j] = both_halves(__fmaf_rn(a.scale, sum[C + i + j], __fmaf_rn(a.linear, g, d)));
                }
            }
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 32; ++j) sum[C + j] = both_halves(__fmul_rn(sum[C + j], a.scale));
        }
        const int32_t x = (int32_t)col, y = (int32_t)(b * a.pad_d + row0);
        put_rows<false, C, BUFFERS>(&maps.d[0], sum, x, y, stage, lane);
        put_rows<true, C, BUFFERS>(&maps.d[1], sum, x, y, stage + (BUFFERS > 1 ? 2048 : 0), lane);
        if (mirrored) {
            if constexpr (BUFFERS == 2) {
                const int32_t xt = (int32_t)row0, yt = (int32_t)(b * a.t.pad_rows + col);
                put_turned_staged<false, C, BUFFERS>(&maps.t[0], sum, xt, yt, stage, lane);
                put_turned_staged<true, C, BUFFERS>(&maps.t[1], sum, xt, yt, stage + 2048, lane);
            } else {
                put_turned<C>(a.t, sum, b, row0, col, a.rows, a.cols, lane);
            }
        }
    }
}

// T: type of kLast's output.
template <uint32_t COLS, bool SPLIT, int KIND, typename T>
__global__ void __launch_bounds__(kThreads, 1) ortho_product_kernel(const __grid_constant__ OrthoMaps maps, const __grid_constant__ OrthoArgs a) {
    static_assert(!SPLIT || COLS == 128, "the exchange is laid out for 128 columns");
    using G = Geom<COLS, SPLIT>;
    constexpr uint32_t kWide = COLS / 4;                   // columns a warp
    extern __shared__ unsigned char dyn[];
    __shared__ volatile uint32_t sh_tmem, sh_failed;
    const uint32_t data = (smem_u32(dyn) + 1023u) & ~1023u;
    unsigned char* stages = dyn + (data - smem_u32(dyn));
    const uint32_t bars = data + G::kSmem - 1024 - 256;
    const auto full = [&](uint32_t s) { return bars + 16u * s; };
    const auto empty = [&](uint32_t s) { return bars + 16u * s + 8u; };
    constexpr uint32_t kChunk = G::kChunk, kSums = G::kSums, kStages = G::kStages;
    const uint32_t acc_full = bars + 16u * kStages, acc_empty = acc_full + 8u * kSums, drain = acc_empty + 8u * kSums, ready = drain + 16u;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, in_cluster = cluster_rank();
    const uint32_t rank = in_cluster & 1u, even = in_cluster & ~1u;            // the pair's CTA that issues
    const uint32_t part = SPLIT ? in_cluster >> 1 : 0, parts = SPLIT ? a.split : 1;
    const uint32_t unit = (blockIdx.x >> 1) / parts, units = (gridDim.x >> 1) / parts;
    const Tiles tiles(a, COLS);
    const uint32_t all_blocks = (uint32_t)((a.k + kBlock - 1) / kBlock), first = all_blocks * part / parts, blocks = all_blocks * (part + 1) / parts - first;

    if (threadIdx.x == 0) {
        sh_failed = 0;
        for (uint32_t s = 0; s < kStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (uint32_t i = 0; i < kSums; ++i) {
            mbar_init(acc_full + 8 * i, 1);
            mbar_init(acc_empty + 8 * i, 32);              // sixteen warps of either CTA
        }
        mbar_init(drain, 1);
        mbar_init(drain + 8, 1);
        mbar_init(ready, 1);
        mbar_init_fence();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            map_prefetch(&maps.p[i]);
            map_prefetch(&maps.q[i]);
            if (KIND != kLast) map_prefetch(&maps.d[i]);
            if (KIND != kLast && SPLIT) map_prefetch(&maps.t[i]);
        }
    }
    cluster_sync_all();
    grid_wait();
    if (warp == 17) {                                      // tensor memory is taken only now: see the 8-bit products
        tmem_alloc<2>(smem_u32((const void*)&sh_tmem), 512);
        if (rank == 1 && lane == 0) cluster_arrive(cluster_map(ready, even));
    }
    if (warp != 16) {
        umma_fence_before();
        asm volatile("bar.sync 1, 576;" ::: "memory");     // the eighteen warps that use it
        umma_fence_after();
        grid_go();
    }

    if (warp == 16 && lane == 0) {
        // ---- feed: this CTA's rows of either factor, completion counted on the even CTA's barrier
        uint32_t it = 0, s = 0, parity = 1;
        bool ok = true;
        for (uint32_t t = unit; ok && t < tiles.count; t += units) {
            uint32_t b, tm, tn;
            tiles.at(t, b, tm, tn);
            const int32_t yp = (int32_t)(b * a.pad_p + tm * 256 + rank * 128), yq = (int32_t)(b * a.pad_q + tn * COLS + rank * (COLS / 2));
            for (uint32_t kb = first; kb < first + blocks; ++kb, ++it) {
                if (it >= kStages && !mbar_wait(empty(s), parity)) { ok = false; break; }
                if (rank == 0) mbar_expect_tx(full(s), 2 * G::kStage);
                const uint32_t dst = data + s * G::kStage, bar = cluster_map(full(s), even);
                const int32_t x = (int32_t)(kb * kBlock);
                tile_load<2>(dst, &maps.p[0], x, yp, bar);
                tile_load<2>(dst + kBox, &maps.p[1], x, yp, bar);
                tile_load<2>(dst + 2 * kBox, &maps.q[0], x, yq, bar);
                tile_load<2>(dst + 2 * kBox + G::kQ, &maps.q[1], x, yq, bar);
                if (++s == kStages) { s = 0; parity ^= 1u; }
            }
        }
        if (!ok) {                                         // the odd CTA cannot see its copies land: leave them a millisecond
            sh_failed = 1;
            for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        }
        // nobody leaves before the copies have landed and the last releases of the stages have arrived
        for (uint32_t j = it > kStages ? it - kStages : 0; j < it; ++j) {
            if (rank == 0) (void)mbar_wait(full(j % kStages), (j / kStages) & 1u);
            if (ok && !mbar_wait(empty(j % kStages), (j / kStages) & 1u)) ok = false;
        }
    } else if (warp >= 17 && warp < 17 + G::kIssuers && lane == 0 && rank == 0) {
        // ---- issue
        constexpr uint32_t idesc = umma_idesc_f16(256, COLS);
        const uint16_t both = (uint16_t)(3u << even);
        const uint32_t mine = warp - 17;
        uint32_t it = 0, n_acc = 0;                        // blocks and sums so far, the other warp's too
        bool ok = mbar_wait(ready, 0);                     // the odd CTA has its tensor memory
        for (uint32_t t = unit; ok && t < tiles.count; t += units) {
            for (uint32_t k0 = 0; ok && k0 < blocks; k0 += kChunk, ++n_acc) {
                const uint32_t acc = n_acc % kSums, use = n_acc / kSums, into = sh_tmem + acc * COLS, n = blocks - k0 < kChunk ? blocks - k0 : kChunk;
                if (n_acc % G::kIssuers != mine) {
                    it += n;
                    continue;
                }
                if (use > 0 && !mbar_wait(acc_empty + 8 * acc, (use - 1) & 1u)) { ok = false; break; }
                umma_fence_after();
                for (uint32_t kb = 0; kb < n; ++kb, ++it) {
                    const uint32_t s = it % kStages;
                    if (!mbar_wait(full(s), (it / kStages) & 1u)) { ok = false; break; }
                    umma_fence_after();
                    const uint32_t at = data + s * G::kStage;
                    const uint64_t ph = umma_desc(at), pl = umma_desc(at + kBox), qh = umma_desc(at + 2 * kBox), ql = umma_desc(at + 2 * kBox + G::kQ);
#pragma unroll
                    for (int j = 0; j < 4; ++j) umma_f16_pair(into, ph + 2 * j, ql + 2 * j, idesc, kb > 0 || j > 0);
#pragma unroll
                    for (int j = 0; j < 4; ++j) umma_f16_pair(into, pl + 2 * j, qh + 2 * j, idesc, true);
#pragma unroll
                    for (int j = 0; j < 4; ++j) umma_f16_pair(into, ph + 2 * j, qh + 2 * j, idesc, true);
                    umma_commit_pair(empty(s), both);
                }
                if (ok) umma_commit_pair(acc_full + 8 * acc, both);
            }
        }
        if (!ok) {
            sh_failed = 1;
            umma_commit_pair(drain + 8 * mine, (uint16_t)(1u << even));
            (void)mbar_wait(drain + 8 * mine, 0);
        }
        // the hand-backs that nothing else waits for come from the other CTA too: they arrive before this one may leave
        for (uint32_t j = n_acc > kSums ? n_acc - kSums : 0; ok && j < n_acc; ++j)
            if (j % G::kIssuers == mine) (void)mbar_wait(acc_empty + 8 * (j % kSums), (j / kSums) & 1u);
    }
    __syncwarp();
    unsigned char* stage = stages + kStages * G::kStage + (SPLIT ? warp & 7 : warp) * G::kStaging;     // (of eight warps in a row eight write)
    const uint32_t quad = warp & 3, group = warp >> 2, row_in = rank * 128 + quad * 32;
    uint32_t n_acc = 0;
    bool ok = true;
    // A tile's sums, chunk by chunk as they come; a failure hands nothing back and shows as NaN.
    float sum[kWide];
    const auto add_up = [&] {
        for (uint32_t k0 = 0; k0 < blocks; k0 += kChunk, ++n_acc) {
            const uint32_t acc = n_acc % kSums, use = n_acc / kSums;
            if (ok && !mbar_wait(acc_full + 8 * acc, use & 1u)) ok = false;
            ok = __all_sync(kFullMask, ok && !sh_failed);
            umma_fence_after();
            if (!ok) continue;
#pragma unroll
            for (uint32_t c = 0; c < kWide; c += 16) {
                uint32_t r[16];
                tmem_ld16(sh_tmem + ((quad * 32) << 16) + acc * COLS + group * kWide + c, r);
                tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; j += 2) {
                    const float2 two = make_float2(__uint_as_float(r[j]), __uint_as_float(r[j + 1]));
                    const float2 all = k0 == 0 ? two : __fadd2_rn(make_float2(sum[c + j], sum[c + j + 1]), two);
                    sum[c + j] = all.x;
                    sum[c + j + 1] = all.y;
                }
            }
            umma_fence_before();
            __syncwarp();
            if (lane == 0) cluster_arrive(cluster_map(acc_empty + 8 * acc, even));
        }
    };
    if constexpr (!SPLIT) {
        if (warp < 16) {
            for (uint32_t t = unit; t < tiles.count; t += units) {
                uint32_t b, tm, tn;
                tiles.at(t, b, tm, tn);
                const uint64_t row0 = (uint64_t)tm * 256 + row_in, col0 = (uint64_t)tn * COLS + group * kWide;
                add_up();
                if (!ok) {
#pragma unroll
                    for (uint32_t j = 0; j < kWide; ++j) sum[j] = CUDART_NAN_F;
                }
                if (row0 >= a.rows) continue;
                const bool mirrored = KIND == kApply || tn < tiles.ratio * tm;
                finish<KIND, T, 0, G::kBuffers>(maps, a, sum, b, row0, col0, mirrored, stage, lane);
                if constexpr (COLS == 256) finish<KIND, T, 32, G::kBuffers>(maps, a, sum, b, row0, col0 + 32, mirrored, stage, lane);
            }
            if (KIND != kLast && lane == 0) tile_store_wait_all();
        }
        __syncwarp();
        __syncthreads();
        cluster_meet_all();                                // the odd CTA's memory is read until the last instruction of the even one
    } else {
        // ---- one tile: leave the other pairs their columns in shared memory, then add up and write out one's own
        const uint32_t cols = 128 / parts, mine = part * cols;
        float4* sums = reinterpret_cast<float4*>(stages);  // [four columns][row]: a warp's access is contiguous; every copy has
        uint32_t b, tm, tn;                                // landed and every instruction has read its operands
        tiles.at(unit, b, tm, tn);
        const uint64_t row0 = (uint64_t)tm * 256 + row_in, col0 = (uint64_t)tn * COLS + group * 32;
        const bool own = warp < 16 && group * 32 >= mine && group * 32 < mine + cols && row0 < a.rows && col0 < a.cols;
        if (warp < 16) {
            add_up();
            if (!ok) sh_failed = 1;
            if (group * 32 < mine || group * 32 >= mine + cols) {
                float4* to = sums + group * 8 * 128 + quad * 32 + lane;
#pragma unroll
                for (int j = 0; j < 8; ++j) to[j * 128] = make_float4(sum[4 * j], sum[4 * j + 1], sum[4 * j + 2], sum[4 * j + 3]);
            }
        }
        __syncwarp();
        cluster_sync_all();
        if (own) {
            const uint32_t from = data + (group * 8 * 128 + quad * 32 + lane) * 16;
            ok = cluster_all_zero(smem_u32((const void*)&sh_failed), 2 * parts);
#pragma unroll 1
            for (uint32_t q = 1; q < parts; ++q) {         // (in the same order each time, not in that of the parts)
                const uint32_t at = cluster_map(from, ((part + q) & (parts - 1)) * 2 + rank);
                int4 v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = cluster_ld4(at + j * 2048);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    sum[4 * j] = __fadd_rn(sum[4 * j], __int_as_float(v[j].x));
                    sum[4 * j + 1] = __fadd_rn(sum[4 * j + 1], __int_as_float(v[j].y));
                    sum[4 * j + 2] = __fadd_rn(sum[4 * j + 2], __int_as_float(v[j].z));
                    sum[4 * j + 3] = __fadd_rn(sum[4 * j + 3], __int_as_float(v[j].w));
                }
            }
        }
        __syncwarp();
        cluster_arrive_all();                              // done with the others' sums
        if (own) {
            if (!ok) {
#pragma unroll
                for (uint32_t j = 0; j < kWide; ++j) sum[j] = CUDART_NAN_F;
            }
            finish<KIND, T, 0, G::kBuffers>(maps, a, sum, b, row0, col0, KIND == kApply || tn < tiles.ratio * tm, stage, lane);
            if (KIND != kLast && lane == 0) tile_store_wait_all();
        }
        __syncwarp();
        cluster_wait_all();                                // nobody leaves while its sums are being read
    }
    if (warp == 17) tmem_free<2>(sh_tmem, 512);
}

// ---- host ------------------------------------------------------------------------------------------
// The batch's matrices one below the other; boxes to load are 64 columns x `load` rows, boxes to store (load = 0) 32 x 32.
bool make_map(CUtensorMap* map, const __half* m, const Halves& h, uint64_t batch, uint32_t load) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {h.cols, h.pad_rows * batch}, strides[1] = {h.ld * 2};
    const cuuint32_t boxes[2] = {load ? 64u : 32u, load ? load : 32u}, steps[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<__half*>(m), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  load ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, load ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_NONE,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool make_maps(CUtensorMap (&maps)[2], const Halves& h, uint64_t batch, uint32_t load) {
    return make_map(&maps[0], h.hi, h, batch, load) && make_map(&maps[1], h.lo, h, batch, load);
}

template <uint32_t COLS, bool SPLIT, int KIND, typename T> cudaError_t launch_product_as(const OrthoMaps& maps, const OrthoArgs& a, uint64_t tiles, cudaStream_t st) {
    static PerDevice<bool> done;
    const auto kernel = ortho_product_kernel<COLS, SPLIT, KIND, T>;
    const int slot = device_slot();
    if (slot < 0 || !done.v[slot]) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Geom<COLS, SPLIT>::kSmem);
        if (e != cudaSuccess) return e;
        if (slot >= 0) done.v[slot] = true;
    }
    const uint64_t pairs = (uint64_t)sm_count_now() / 2, units = SPLIT ? tiles * a.split : tiles < pairs ? tiles : pairs;
    return launch_layer(kernel, (unsigned)(2 * units), kThreads, Geom<COLS, SPLIT>::kSmem, 2 * a.split, st, maps, a);
}
uint64_t count_tiles(uint64_t batch, uint64_t rows, uint64_t cols, bool symmetric, uint64_t width) {
    const uint64_t down = (rows + 255) / 256, across = (cols + width - 1) / width, ratio = 256 / width;
    return batch * (symmetric ? ratio * (down * (down + 1) / 2) - (down * ratio - across) : down * across);
}
// How a product is cut.
struct Cut {
    uint32_t width, split;
    uint64_t tiles;
};
// The tiles whose waves over the pairs take less time (about 2000 and 1150 cycles a block of the contraction); narrow ones that leave pairs idle
// have their contraction split, two blocks at least to a part, as long as all clusters run at once (counted on a B200: 74 pairs, 33
// clusters of two, 16 of four).
Cut cut_product(uint64_t batch, uint64_t rows, uint64_t cols, uint64_t k, bool symmetric) {
    const uint64_t pairs = (uint64_t)sm_count_now() / 2, blocks = (k + kBlock - 1) / kBlock;
    const uint64_t wide = count_tiles(batch, rows, cols, symmetric, 256), narrow = count_tiles(batch, rows, cols, symmetric, 128);
    if ((wide + pairs - 1) / pairs * 2000 <= (narrow + pairs - 1) / pairs * 1150) return {256, 1, wide};
    const uint32_t split = narrow <= 16 && blocks >= 8 ? 4 : narrow <= 33 && blocks >= 4 ? 2 : 1;
    return {128, split, narrow};
}
// Cycles that a product takes about: its waves, and 7 us for a launch, its first copies and its output.
uint64_t product_cycles(uint64_t batch, uint64_t rows, uint64_t cols, uint64_t k, bool symmetric) {
    const Cut cut = cut_product(batch, rows, cols, k, symmetric);
    const uint64_t pairs = (uint64_t)sm_count_now() / 2;
    return (cut.tiles + pairs - 1) / pairs * ((k + kBlock - 1) / kBlock) * (cut.width == 256 ? 2000 : 1150) / cut.split + 13000;
}
template <int KIND, typename T> cudaError_t launch_product(const OrthoMaps& maps, const OrthoArgs& a, const Cut& cut, cudaStream_t st) {
    if (cut.width == 256) return launch_product_as<256, false, KIND, T>(maps, a, cut.tiles, st);
    return cut.split > 1 ? launch_product_as<128, true, KIND, T>(maps, a, cut.tiles, st) : launch_product_as<128, false, KIND, T>(maps, a, cut.tiles, st);
}

uint64_t up(uint64_t n, uint64_t to) { return (n + to - 1) / to * to; }
uint64_t halves_bytes(uint64_t batch, uint64_t rows, uint64_t cols) { return 2 * up(batch * up(rows, 128) * up(cols, 64) * 2, 256); }
struct Carver {
    unsigned char* at;
    Halves take(uint64_t batch, uint64_t rows, uint64_t cols) {
        const uint64_t half = halves_bytes(batch, rows, cols) / 2;
        Halves h{reinterpret_cast<__half*>(at), reinterpret_cast<__half*>(at + half), rows, cols, up(rows, 128), up(cols, 64)};
        at += 2 * half;
        return h;
    }
};

// The largest |a x + b x^3 + c x^5| and |a + b x^2 + c x^4| over [0, most]: both at an end or where a derivative vanishes.
void polynomial_bounds(double a, double b, double c, double most, double& value, double& factor) {
    const auto at = [&](double x2) {
        if (!(x2 >= 0.0)) return;
        const double x = std::sqrt(x2) < most ? std::sqrt(x2) : most, y = x * x;
        factor = std::fmax(factor, std::fabs(a + (b + c * y) * y));
        value = std::fmax(value, std::fabs(x * (a + (b + c * y) * y)));
    };
    value = factor = 0.0;
    at(0.0);
    at(most * most);
    if (c != 0.0) {
        const double root = 9.0 * b * b - 20.0 * a * c;    // a + 3 b y + 5 c y^2 = 0
        if (root >= 0.0) {
            at((-3.0 * b + std::sqrt(root)) / (10.0 * c));
            at((-3.0 * b - std::sqrt(root)) / (10.0 * c));
        }
        at(-b / (2.0 * c));                                // b + 2 c y = 0
    } else if (b != 0.0) {
        at(-a / (3.0 * b));
    }
}

}  // namespace
}  // namespace tng

using namespace tng;

extern "C" {

// Three more matrices of the shorter side for sizes that may take several steps at once.
static bool may_group(uint64_t s, uint64_t l) { return s >= 1024 && l >= 2 * s; }

size_t tng_orthogonalize_scratch_bytes(uint64_t batch, uint64_t rows, uint64_t cols) {
    if (batch == 0 || rows == 0 || cols == 0) return 256;
    const uint64_t s = rows < cols ? rows : cols, l = rows < cols ? cols : rows;
    return (size_t)(batch * kNormBlocks * 8 + halves_bytes(batch, s, l) + 2 * halves_bytes(batch, l, s) + (may_group(s, l) ? 5 : 2) * halves_bytes(batch, s, s));
}

tng_status tng_orthogonalize(const void* v_dev, tng_dtype type, uint64_t batch, uint64_t rows, uint64_t cols, uint64_t ldv, uint64_t stride,
                             uint32_t steps, float a, float b, float c, void* out_dev, tng_dtype out_type, uint64_t ldo, uint64_t out_stride,
                             void* scratch_dev, void* stream) {
    if (!type_ok(type) || !type_ok(out_type) || rows < 1 || cols < 1 || rows >= (1u << 30) || cols >= (1u << 30) || batch > 65535 || steps < 1 || steps > 64 || !std::isfinite(a) ||
        !std::isfinite(b) || !std::isfinite(c))
        return TNG_ERR_INVALID_ARG;
    // what the factors may grow to, step by step (2^-10 for rounding)
    double most = 1.0, factors[64];
    for (uint32_t i = 0; i < steps; ++i) {
        double value, factor;
        polynomial_bounds(a, b, c, most, value, factor);
        if (!(value <= kMostX && factor <= kMostB)) return TNG_ERR_INVALID_ARG;
        most = std::fmax(value, 0.0) * (1.0 + 0x1p-10);
        factors[i] = factor * (1.0 + 0x1p-10);
    }
    if (batch == 0) return TNG_OK;
    const uint64_t s = rows < cols ? rows : cols, l = rows < cols ? cols : rows;
    if (s > 64 * 65535 || batch * up(l, 128) >= (1ull << 31) || (batch * up(s, 128) / 128) * (up(l, 128) / 128) >= (1ull << 31)) return TNG_ERR_INVALID_ARG;
    if (!matrix_ok(v_dev, type, cols, ldv) || !matrix_ok(out_dev, out_type, cols, ldo) || (batch > 1 && out_stride == 0) || !scratch_dev || !aligned(scratch_dev, 256)) return TNG_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    unsigned char* at = static_cast<unsigned char*>(scratch_dev);
    double* part = reinterpret_cast<double*>(at);
    Carver carve{at + batch * kNormBlocks * 8};
    const Halves x = carve.take(batch, s, l), g = carve.take(batch, s, s), poly = carve.take(batch, s, s);
    const Halves xt = carve.take(batch, l, s), xt2 = carve.take(batch, l, s);
    const bool tall = rows > cols;
    cudaError_t e = with_type(type, [&](auto t) {
        using T = decltype(t);
        const T* v = static_cast<const T*>(v_dev);
        cudaError_t err = launch_layer(ortho_norm_kernel<T>, dim3(kNormBlocks, (unsigned)batch), kNormThreads, 0, 1, st, v, rows, cols, ldv, stride, part);
        if (err != cudaSuccess) return err;
        const dim3 grid((unsigned)((l + 63) / 64), (unsigned)((s + 63) / 64), (unsigned)batch);
        return launch_layer(ortho_split_kernel<T>, grid, 256, 0, 1, st, v, ldv, stride, static_cast<const double*>(part), tall ? xt : x, tall ? x : xt);
    });
    if (e != cudaSuccess) return layer_status(e);
    if (may_group(s, l) && out_type != TNG_F32) {
        const uint32_t groups = (steps + kMostGroup - 1) / kMostGroup;
        const uint64_t square = product_cycles(batch, s, s, s, true), once = product_cycles(batch, s, s, l, true) + product_cycles(batch, s, l, s, false);
        // (the products of the shorter side's size: steps + 3 (steps - groups))
        if (groups * once + (4 * steps - 3 * groups) * square < steps * (once + square)) {
            Halves t = carve.take(batch, s, s), q[2] = {carve.take(batch, s, s), carve.take(batch, s, s)};
            OrthoArgs args = {};
            args.batch = (uint32_t)batch;
            // a symmetric product of the shorter side's size, or G itself
            const auto symmetric = [&](auto kind, const Halves& p, const Halves& o, const Halves& d, uint64_t k, float scale) {
                const Cut cut = cut_product(batch, s, s, k, true);
                OrthoMaps m = {};
                if (!make_maps(m.p, p, batch, 128) || !make_maps(m.q, o, batch, cut.width / 2) || !make_maps(m.d, d, batch, 0) || (cut.split > 1 && !make_maps(m.t, d, batch, 0))) return cudaErrorNotSupported;
                args.rows = args.cols = s;
                args.k = k;
                args.pad_p = args.pad_q = args.pad_d = x.pad_rows;
                args.t = d;
                args.symmetric = 1;
                args.split = cut.split;
                args.scale = scale;
                return launch_product<decltype(kind)::value, float>(m, args, cut, st);
            };
            using Gram = std::integral_constant<int, kGram>;
            using Poly = std::integral_constant<int, kPoly>;
            args.linear = b * (kScaleB / kScaleG);
            args.diagonal = a * kScaleB;
            args.g = g;
            for (uint32_t group = 0, i = 0; group < groups && e == cudaSuccess; ++group) {
                const uint32_t end = steps * (group + 1) / groups;
                e = symmetric(Gram(), x, x, g, l, kScaleG / (kScaleX * kScaleX));
                // Q, the product of the group's Bs: the first B itself; as large a power of two as its bound leaves room for
                uint32_t now = 0;
                float scale_q = kScaleB;
                double bound = 1.0;
                for (uint32_t first = i; i < end && e == cudaSuccess; ++i) {
                    const Halves& by = i == first ? q[0] : poly;
                    bound *= factors[i];
                    e = symmetric(Poly(), g, g, by, s, c * (kScaleB / (kScaleG * kScaleG)));
                    if (i > first && e == cudaSuccess) {
                        const float scale = std::fmin(kScaleB, (float)std::exp2(std::floor(std::log2(60000.0 / std::fmax(bound, 1.0)))));
                        e = symmetric(Gram(), poly, q[now], q[now ^ 1], s, scale / (kScaleB * scale_q));
                        scale_q = scale;
                        now ^= 1;
                    }
                    if (i + 1 < end && e == cudaSuccess) {         // G <- B (B G)
                        e = symmetric(Gram(), by, g, t, s, kScaleG / (kScaleB * kScaleG));
                        if (e == cudaSuccess) e = symmetric(Gram(), by, t, g, s, kScaleG / (kScaleB * kScaleG));
                    }
                }
                if (e != cudaSuccess) break;
                const bool final = group + 1 == groups, flip = final && tall;
                const Halves &from = group & 1 ? xt2 : xt, &to = group & 1 ? xt : xt2;
                const Cut cut = final ? cut_product(batch, rows, cols, s, false) : cut_product(batch, s, l, s, false);
                OrthoMaps m = {};
                if (!make_maps(m.p, flip ? from : q[now], batch, 128) || !make_maps(m.q, flip ? q[now] : from, batch, cut.width / 2) ||
                    (!final && (!make_maps(m.d, x, batch, 0) || (cut.split > 1 && !make_maps(m.t, to, batch, 0)))))
                    return TNG_ERR_CUDA;
                OrthoArgs last = args;
                last.symmetric = 0;
                last.k = s;
                last.split = cut.split;
                last.rows = final ? rows : s;
                last.cols = final ? cols : l;
                last.pad_p = flip ? xt.pad_rows : x.pad_rows;
                last.pad_q = flip ? x.pad_rows : xt.pad_rows;
                last.t = to;
                last.scale = 1.f / (final ? scale_q * kScaleX : scale_q);
                last.out = out_dev;
                last.ldo = ldo;
                last.stride = out_stride;
                e = final ? with_type(out_type, [&](auto type_of) { return launch_product<kLast, decltype(type_of)>(m, last, cut, st); })
                          : launch_product<kApply, float>(m, last, cut, st);
            }
            return layer_status(e);
        }
    }

    // The products of a step: G = X X^T, B from G, X <- B X (the last one as the output lies: B X, or X^T B).
    const Cut cut_gram = cut_product(batch, s, s, l, true), cut_poly = cut_product(batch, s, s, s, true);
    const Cut cut_apply = cut_product(batch, s, l, s, false), cut_last = cut_product(batch, rows, cols, s, false);
    const auto maps_of = [&](OrthoMaps& m, const Cut& cut, const Halves& p, const Halves& q, const Halves* d, const Halves* t) {
        return make_maps(m.p, p, batch, 128) && make_maps(m.q, q, batch, cut.width / 2) && (!d || make_maps(m.d, *d, batch, 0)) &&
               (!t || cut.split == 1 || make_maps(m.t, *t, batch, 0));
    };
    OrthoMaps gram = {}, square = {}, apply[2] = {}, last = {};
    const Halves& xt_last = (steps - 1) & 1 ? xt2 : xt;
    if (!maps_of(gram, cut_gram, x, x, &g, &g) || !maps_of(square, cut_poly, g, g, &poly, &poly) ||
        (steps > 1 && !maps_of(apply[0], cut_apply, poly, xt, &x, &xt2)) || (steps > 2 && !maps_of(apply[1], cut_apply, poly, xt2, &x, &xt)) ||
        !(tall ? maps_of(last, cut_last, xt_last, poly, nullptr, nullptr) : maps_of(last, cut_last, poly, xt_last, nullptr, nullptr)))
        return TNG_ERR_CUDA;
    OrthoArgs square_args = {};                            // of both symmetric products
    square_args.batch = (uint32_t)batch;
    square_args.rows = square_args.cols = s;
    square_args.pad_p = square_args.pad_q = square_args.pad_d = x.pad_rows;
    square_args.symmetric = 1;
    square_args.g = g;
    for (uint32_t i = 0; i < steps; ++i) {
        OrthoArgs args = square_args;
        args.split = cut_gram.split;
        args.k = l;
        args.t = g;
        args.scale = kScaleG / (kScaleX * kScaleX);
        e = launch_product<kGram, float>(gram, args, cut_gram, st);
        if (e != cudaSuccess) return layer_status(e);
        args.split = cut_poly.split;
        args.k = s;
        args.t = poly;
        args.scale = c * (kScaleB / (kScaleG * kScaleG));
        args.linear = b * (kScaleB / kScaleG);
        args.diagonal = a * kScaleB;
        e = launch_product<kPoly, float>(square, args, cut_poly, st);
        if (e != cudaSuccess) return layer_status(e);
        args.symmetric = 0;
        if (i + 1 < steps) {
            args.split = cut_apply.split;
            args.cols = l;
            args.pad_q = xt.pad_rows;
            args.t = i & 1 ? xt : xt2;
            args.scale = 1.f / kScaleB;
            e = launch_product<kApply, float>(apply[i & 1], args, cut_apply, st);
        } else {
            args.split = cut_last.split;
            args.rows = rows;
            args.cols = cols;
            (tall ? args.pad_p : args.pad_q) = xt.pad_rows;
            args.scale = 1.f / (kScaleB * kScaleX);
            args.out = out_dev;
            args.ldo = ldo;
            args.stride = out_stride;
            e = with_type(out_type, [&](auto t) { return launch_product<kLast, decltype(t)>(last, args, cut_last, st); });
        }
        if (e != cudaSuccess) return layer_status(e);
    }
    return TNG_OK;
}

}  // extern "C"
