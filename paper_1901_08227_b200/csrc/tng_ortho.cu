// Orthogonalised updates: X = V / |V| (Frobenius), then X <- (a I + b G + c G^2) X with G = X X^T, a few times over.  Every step is an
// odd polynomial of the singular values alone, so that they move towards one while the singular vectors stay.
//
// A step is three products: G = X X^T and B = a I + b G + c G G (both symmetric: only the tiles on and below the diagonal are
// computed, and written twice), then B X.  With s the shorter side and l the longer, 3 s^2 l + s^3 operations.
//
// Accuracy.  Every factor is held as two fp16 numbers, hi + lo, 22 bits together, times a power of two that keeps the bounds below in
// fp16's range and its steps far below the entries; a product is three (hi lo, lo hi, hi hi), lo lo being below 2^-22 of it.
// (bf16 factors alone, 8 bits, would do for the singular values that are near one, but a step multiplies what lies in the
// directions of the small ones by up to a: after five steps rounding noise of 2^-9 has grown by a factor of hundreds there.)  The tensor
// memory's sums lose about half a step of fp32 with every instruction, all in one direction; so they run over kChunk blocks
// of the contraction only, and the chunks are added to nearest in registers.
//
// Bounds (checked on the host for the given coefficients): singular values of X at most 2, so entries of X at most 2, of G 4, and of B
// 15; stored as X 2^14, G 2^13, B 2^12.
#include <math_constants.h>

#include <cmath>

#include "tng_layers.cuh"
#include "tng_umma.cuh"

namespace tng {
namespace {

constexpr float kScaleX = 0x1p14f, kScaleG = 0x1p13f, kScaleB = 0x1p12f;
constexpr double kMostX = 2.0, kMostB = 15.0;

// A matrix held in two halves: `batch` of them, rows rounded up to 128, row stride ld.
struct Halves {
    __half *hi, *lo;
    uint64_t rows, cols, pad_rows, ld;
};

// ---- |V| and its two halves --------------------------------------------------------------------------------
// The sum of squares in 64 bits (no overflow, no underflow, and its rounding does not show), each block's share on its own.
constexpr uint32_t kNormBlocks = 128;
template <typename T>
__global__ void __launch_bounds__(256) ortho_norm_kernel(const T* v, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t stride, double* part) {
    __shared__ double sh[8];
    grid_wait();
    grid_go();
    v += blockIdx.y * stride;
    double s = 0.0;
    for (uint64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* row = v + r * ld;
        for (uint64_t c = threadIdx.x; c < cols; c += 256) {
            const double e = (double)to_f32(row[c]);
            s += e * e;
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(kFullMask, s, d);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) s += sh[i];
        part[blockIdx.y * kNormBlocks + blockIdx.x] = s;
    }
}

__device__ __forceinline__ void split(float v, __half& hi, __half& lo) {
    hi = __float2half_rn(v);
    lo = __float2half_rn(__fsub_rn(v, __half2float(hi)));
}

// V / |V| in two halves, as it lies and transposed.  A block has 64 x 64 elements.
template <typename T>
__global__ void __launch_bounds__(256) ortho_split_kernel(const T* v, uint64_t ld, uint64_t stride, const double* part, const __grid_constant__ Halves as,
                                                          const __grid_constant__ Halves turned) {
    __shared__ __half hi[64][66], lo[64][66];
    __shared__ double total[8];
    grid_wait();
    grid_go();
    const uint32_t b = blockIdx.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double s = threadIdx.x < kNormBlocks ? part[b * kNormBlocks + threadIdx.x] : 0.0;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(kFullMask, s, d);
    if (lane == 0) total[warp] = s;
    __syncthreads();
    const double norm = sqrt((total[0] + total[1]) + (total[2] + total[3]));
    // (a norm that is not finite makes all of the matrix NaN, a zero one leaves it zero)
    const double f = norm == 0.0 ? 0.0 : norm < (double)CUDART_INF ? (double)kScaleX / norm : (double)CUDART_NAN_F;
    const uint64_t r0 = (uint64_t)blockIdx.y * 64, c0 = (uint64_t)blockIdx.x * 64;
    v += b * stride;
    for (uint32_t i = threadIdx.x; i < 4096; i += 256) {
        const uint64_t r = r0 + (i >> 6), c = c0 + (i & 63);
        const float e = r < as.rows && c < as.cols ? (float)((double)to_f32(v[r * ld + c]) * f) : 0.f;
        split(e, hi[i >> 6][i & 63], lo[i >> 6][i & 63]);
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 4096; i += 256) {
        const uint32_t p = i >> 6, q = i & 63;
        if (r0 + p < as.rows && c0 + q < as.cols) {
            const uint64_t at = (b * as.pad_rows + r0 + p) * as.ld + c0 + q;
            as.hi[at] = hi[p][q];
            as.lo[at] = lo[p][q];
        }
        if (c0 + p < turned.rows && r0 + q < turned.cols) {
            const uint64_t at = (b * turned.pad_rows + c0 + p) * turned.ld + r0 + q;
            turned.hi[at] = hi[q][p];
            turned.lo[at] = lo[q][p];
        }
    }
}

// ---- products --------------------------------------------------------------------------------------------
// D = P Q^T of two matrices in halves, contraction along the rows of both.  PAIR: 256 x 256 tiles of two SMs, else 128 x 128 of one:
// either way a CTA copies 128 rows of each factor, both halves, 64 KB a stage of 64 of the contraction (12 instructions), and
// three stages are under way.  Warps: 0-15 add up and write out (a quarter of the rows and of the columns each), 16 feeds, 17 issues.
enum Kind { kGram = 0, kPoly = 1, kApply = 2, kLast = 3 };
constexpr int kThreads = 576;
constexpr uint32_t kBox = 128 * 128, kStage = 4 * kBox, kStages = 3, kStaging = 2048, kBlock = 64, kChunk = 1;
constexpr uint32_t kSmem = 1024 + kStages * kStage + 16 * kStaging + 256;
static_assert(kSmem <= 227 * 1024, "shared memory of a CTA");

struct OrthoMaps {
    CUtensorMap p[2], q[2], d[2], t[2];   // hi and lo of the factors, of D and of its transpose
};
struct OrthoArgs {
    uint64_t rows, cols, k;         // of D, and the contraction
    uint64_t pad_p, pad_q, pad_d, pad_t;   // rows from one matrix of the batch to the next
    uint32_t batch, symmetric;
    float scale, linear, diagonal;  // D = scale * sum (+ linear * g + diagonal on the diagonal: kPoly)
    Halves g;                       // kPoly: the factor itself
    void* out;                      // kLast
    uint64_t ldo, stride;
};

// A launch's tiles: by matrix, then by rows of tiles.  Symmetric products: those on and below the diagonal.
struct Tiles {
    uint32_t down, across, per, count, symmetric;
    __device__ __forceinline__ Tiles(const OrthoArgs& a, uint32_t edge) {
        down = (uint32_t)((a.rows + edge - 1) / edge);
        across = (uint32_t)((a.cols + edge - 1) / edge);
        symmetric = a.symmetric;
        per = symmetric ? down * (down + 1) / 2 : down * across;
        count = per * a.batch;
    }
    __device__ __forceinline__ void at(uint32_t t, uint32_t& b, uint32_t& tm, uint32_t& tn) const {
        b = t / per;
        t -= b * per;
        if (symmetric) {
            tm = (uint32_t)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
            while (tm * (tm + 1) / 2 > t) --tm;
            while ((tm + 1) * (tm + 2) / 2 <= t) ++tm;
            tn = t - tm * (tm + 1) / 2;
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
template <bool LO, uint32_t C, uint32_t N>
__device__ __forceinline__ void put_rows(const CUtensorMap* map, const float (&v)[N], int32_t x, int32_t y, unsigned char* stage, uint32_t lane) {
    if (lane == 0) tile_store_wait_read<0>();
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
template <bool LO, uint32_t C, uint32_t N>
__device__ __forceinline__ void put_turned(const CUtensorMap* map, const float (&v)[N], int32_t x, int32_t y, unsigned char* stage, uint32_t lane) {
    if (lane == 0) tile_store_wait_read<0>();
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

// A warp's 32 columns from C of its sums, finished and written: see ortho_product_kernel.
template <int KIND, typename T, uint32_t C, uint32_t N>
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
            for (uint32_t i = 0; i < 32; i += 8) {
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
        const int32_t x = (int32_t)col, y = (int32_t)(b * a.pad_d + row0), xt = (int32_t)row0, yt = (int32_t)(b * a.pad_t + col);
        put_rows<false, C>(&maps.d[0], sum, x, y, stage, lane);
        put_rows<true, C>(&maps.d[1], sum, x, y, stage, lane);
        if (mirrored) {
            put_turned<false, C>(&maps.t[0], sum, xt, yt, stage, lane);
            put_turned<true, C>(&maps.t[1], sum, xt, yt, stage, lane);
        }
    }
}

// T: type of kLast's output.
template <bool PAIR, int KIND, typename T>
__global__ void __launch_bounds__(kThreads, 1) ortho_product_kernel(const __grid_constant__ OrthoMaps maps, const __grid_constant__ OrthoArgs a) {
    constexpr int GROUP = PAIR ? 2 : 1;
    constexpr uint32_t kEdge = PAIR ? 256 : 128, kWide = kEdge / 4;         // columns a warp
    extern __shared__ unsigned char dyn[];
    __shared__ volatile uint32_t sh_tmem, sh_failed;
    const uint32_t data = (smem_u32(dyn) + 1023u) & ~1023u;
    const uint32_t bars = data + kStages * kStage + 16 * kStaging;
    const auto full = [&](uint32_t s) { return bars + 16u * s; };
    const auto empty = [&](uint32_t s) { return bars + 16u * s + 8u; };
    const uint32_t acc_full = bars + 16u * kStages, acc_empty = acc_full + 16u, drain = acc_full + 32u, ready = acc_full + 40u;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = PAIR ? cluster_rank() : 0u;
    const uint32_t unit = PAIR ? blockIdx.x >> 1 : blockIdx.x, units = PAIR ? gridDim.x >> 1 : gridDim.x;
    const Tiles tiles(a, kEdge);
    const uint32_t blocks = (uint32_t)((a.k + kBlock - 1) / kBlock);

    if (threadIdx.x == 0) {
        sh_failed = 0;
        for (uint32_t s = 0; s < kStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (uint32_t i = 0; i < 2; ++i) {
            mbar_init(acc_full + 8 * i, 1);
            mbar_init(acc_empty + 8 * i, 16 * GROUP);      // sixteen warps of each CTA
        }
        mbar_init(drain, 1);
        mbar_init(ready, 1);
        mbar_init_fence();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            map_prefetch(&maps.p[i]);
            map_prefetch(&maps.q[i]);
        }
    }
    if (PAIR) cluster_sync_all();
    else __syncthreads();
    grid_wait();
    if (warp == 17) {                                      // tensor memory is taken only now: see the 8-bit products
        tmem_alloc<GROUP>(smem_u32((const void*)&sh_tmem), 2 * kEdge);
        if (PAIR && rank == 1 && lane == 0) cluster_arrive(cluster_map(ready, 0));
    }
    if (warp != 16) {
        umma_fence_before();
        asm volatile("bar.sync 1, 544;" ::: "memory");     // the seventeen warps that use it
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
            const int32_t yp = (int32_t)(b * a.pad_p + tm * kEdge + rank * 128), yq = (int32_t)(b * a.pad_q + tn * kEdge + rank * 128);
            for (uint32_t kb = 0; kb < blocks; ++kb, ++it) {
                if (it >= kStages && !mbar_wait(empty(s), parity)) { ok = false; break; }
                if (rank == 0) mbar_expect_tx(full(s), GROUP * kStage);
                const uint32_t dst = data + s * kStage, bar = PAIR ? cluster_map(full(s), 0) : full(s);
                const int32_t x = (int32_t)(kb * kBlock);
                tile_load<GROUP>(dst, &maps.p[0], x, yp, bar);
                tile_load<GROUP>(dst + kBox, &maps.p[1], x, yp, bar);
                tile_load<GROUP>(dst + 2 * kBox, &maps.q[0], x, yq, bar);
                tile_load<GROUP>(dst + 3 * kBox, &maps.q[1], x, yq, bar);
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
    } else if (warp == 17 && lane == 0 && rank == 0) {
        // ---- issue
        constexpr uint32_t idesc = umma_idesc_f16(kEdge, kEdge);
        uint32_t s = 0, parity = 0, n_acc = 0;
        bool ok = !PAIR || mbar_wait(ready, 0);            // the odd CTA has its tensor memory
        for (uint32_t t = unit; ok && t < tiles.count; t += units) {
            for (uint32_t k0 = 0; ok && k0 < blocks; k0 += kChunk, ++n_acc) {
                const uint32_t acc = n_acc & 1u, use = n_acc >> 1, into = sh_tmem + acc * kEdge, n = blocks - k0 < kChunk ? blocks - k0 : kChunk;
                if (use > 0 && !mbar_wait(acc_empty + 8 * acc, (use - 1) & 1u)) { ok = false; break; }
                umma_fence_after();
                for (uint32_t kb = 0; kb < n; ++kb) {
                    if (!mbar_wait(full(s), parity)) { ok = false; break; }
                    umma_fence_after();
                    const uint32_t at = data + s * kStage;
                    const uint64_t ph = umma_desc(at), pl = umma_desc(at + kBox), qh = umma_desc(at + 2 * kBox), ql = umma_desc(at + 3 * kBox);
#pragma unroll
                    for (int j = 0; j < 4; ++j) umma_f16<GROUP>(into, ph + 2 * j, ql + 2 * j, idesc, kb > 0 || j > 0);
#pragma unroll
                    for (int j = 0; j < 4; ++j) umma_f16<GROUP>(into, pl + 2 * j, qh + 2 * j, idesc, true);
#pragma unroll
                    for (int j = 0; j < 4; ++j) umma_f16<GROUP>(into, ph + 2 * j, qh + 2 * j, idesc, true);
                    umma_commit_all<GROUP>(empty(s), 3);
                    if (++s == kStages) { s = 0; parity ^= 1u; }
                }
                if (ok) umma_commit_all<GROUP>(acc_full + 8 * acc, 3);
            }
        }
        if (!ok) {
            sh_failed = 1;
            umma_commit_all<GROUP>(drain, 1);
            (void)mbar_wait(drain, 0);
        }
        // the hand-backs that nothing else waits for come from the other CTA too: they arrive before this one may leave
        for (uint32_t j = n_acc > 2 ? n_acc - 2 : 0; j < n_acc; ++j) (void)mbar_wait(acc_empty + 8 * (j & 1u), (j >> 1) & 1u);
    }
    __syncwarp();
    if (warp < 16) {
        // ---- add up and write out: rows 32 quad + lane of this CTA's 128, kWide columns
        unsigned char* stage = dyn + (data - smem_u32(dyn)) + kStages * kStage + warp * kStaging;
        const uint32_t quad = warp & 3, group = warp >> 2;
        uint32_t n_acc = 0;
        bool ok = true;
        for (uint32_t t = unit; t < tiles.count; t += units) {
            uint32_t b, tm, tn;
            tiles.at(t, b, tm, tn);
            const uint64_t row0 = (uint64_t)tm * kEdge + rank * 128 + quad * 32, col0 = (uint64_t)tn * kEdge + group * kWide;
            float sum[kWide];
            for (uint32_t k0 = 0; k0 < blocks; k0 += kChunk, ++n_acc) {
                const uint32_t acc = n_acc & 1u, use = n_acc >> 1;
                if (ok && !mbar_wait(acc_full + 8 * acc, use & 1u)) ok = false;
                ok = __all_sync(kFullMask, ok && !sh_failed);
                umma_fence_after();
                if (ok) {
#pragma unroll
                    for (uint32_t c = 0; c < kWide; c += 16) {
                        uint32_t r[16];
                        tmem_ld16(sh_tmem + ((quad * 32) << 16) + acc * kEdge + group * kWide + c, r);
                        tmem_wait_ld();
                        if (k0 == 0) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) sum[c + j] = __uint_as_float(r[j]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 16; ++j) sum[c + j] = __fadd_rn(sum[c + j], __uint_as_float(r[j]));
                        }
                    }
                    umma_fence_before();
                    __syncwarp();
                    if (lane == 0) cluster_arrive(cluster_map(acc_empty + 8 * acc, 0));    // (a failure hands nothing back)
                }
            }
            if (!ok) {
#pragma unroll
                for (uint32_t j = 0; j < kWide; ++j) sum[j] = CUDART_NAN_F;
            }
            if (row0 >= a.rows) continue;
            const bool mirrored = KIND == kApply || tm != tn;
            finish<KIND, T, 0>(maps, a, sum, b, row0, col0, mirrored, stage, lane);
            if constexpr (PAIR) finish<KIND, T, 32>(maps, a, sum, b, row0, col0 + 32, mirrored, stage, lane);
        }
        if (KIND != kLast && lane == 0) tile_store_wait_all();
    }
    __syncwarp();
    __syncthreads();
    if (PAIR) cluster_meet_all();                          // the odd CTA's memory is read until the last instruction of the even one
    if (warp == 17) tmem_free<GROUP>(sh_tmem, 2 * kEdge);
}

// ---- host ------------------------------------------------------------------------------------------
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
    static const EncodeTiled fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            f = nullptr;
        }
        return reinterpret_cast<EncodeTiled>(f);
    }();
    return fn;
}
// The batch's matrices one below the other; boxes to load are 64 columns x 128 rows, boxes to store 32 x 32.
bool make_map(CUtensorMap* map, const __half* m, const Halves& h, uint64_t batch, bool load) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {h.cols, h.pad_rows * batch}, strides[1] = {h.ld * 2};
    const cuuint32_t boxes[2] = {load ? 64u : 32u, load ? 128u : 32u}, steps[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<__half*>(m), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  load ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, load ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_NONE,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool make_maps(CUtensorMap (&maps)[2], const Halves& h, uint64_t batch, bool load) {
    return make_map(&maps[0], h.hi, h, batch, load) && make_map(&maps[1], h.lo, h, batch, load);
}

template <bool PAIR, int KIND, typename T> cudaError_t launch_product_as(const OrthoMaps& maps, const OrthoArgs& a, cudaStream_t st) {
    static PerDevice<bool> done;
    const auto kernel = ortho_product_kernel<PAIR, KIND, T>;
    const int slot = device_slot();
    if (slot < 0 || !done.v[slot]) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
        if (e != cudaSuccess) return e;
        if (slot >= 0) done.v[slot] = true;
    }
    const uint64_t edge = PAIR ? 256 : 128, down = (a.rows + edge - 1) / edge, across = (a.cols + edge - 1) / edge;
    const uint64_t tiles = a.batch * (a.symmetric ? down * (down + 1) / 2 : down * across), most = (uint64_t)sm_count_now() / (PAIR ? 2 : 1);
    return launch_layer(kernel, (unsigned)((tiles < most ? tiles : most) * (PAIR ? 2 : 1)), kThreads, kSmem, PAIR ? 2 : 1, st, maps, a);
}
// Which tiles: large ones where they keep the pairs busy.
bool takes_pairs(const OrthoArgs& a) {
    const uint64_t down = (a.rows + 255) / 256, across = (a.cols + 255) / 256;
    return a.batch * (a.symmetric ? down * (down + 1) / 2 : down * across) >= (uint64_t)sm_count_now() / 2;
}
template <int KIND, typename T> cudaError_t launch_product(const OrthoMaps& maps, const OrthoArgs& a, cudaStream_t st) {
    return takes_pairs(a) ? launch_product_as<true, KIND, T>(maps, a, st) : launch_product_as<false, KIND, T>(maps, a, st);
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

size_t tng_orthogonalize_scratch_bytes(uint64_t batch, uint64_t rows, uint64_t cols) {
    if (batch == 0 || rows == 0 || cols == 0) return 256;
    const uint64_t s = rows < cols ? rows : cols, l = rows < cols ? cols : rows;
    return (size_t)(batch * kNormBlocks * 8 + halves_bytes(batch, s, l) + 2 * halves_bytes(batch, l, s) + 2 * halves_bytes(batch, s, s));
}

tng_status tng_orthogonalize(const void* v_dev, tng_dtype type, uint64_t batch, uint64_t rows, uint64_t cols, uint64_t ldv, uint64_t stride,
                             uint32_t steps, float a, float b, float c, void* out_dev, tng_dtype out_type, uint64_t ldo, uint64_t out_stride,
                             void* scratch_dev, void* stream) {
    if (!type_ok(type) || !type_ok(out_type) || rows < 1 || cols < 1 || rows >= (1u << 30) || cols >= (1u << 30) || batch > 65535 || steps < 1 || steps > 64 || !std::isfinite(a) ||
        !std::isfinite(b) || !std::isfinite(c))
        return TNG_ERR_INVALID_ARG;
    // what the factors may grow to, step by step (2^-10 for rounding)
    double most = 1.0;
    for (uint32_t i = 0; i < steps; ++i) {
        double value, factor;
        polynomial_bounds(a, b, c, most, value, factor);
        if (!(value <= kMostX && factor <= kMostB)) return TNG_ERR_INVALID_ARG;
        most = std::fmax(value, 0.0) * (1.0 + 0x1p-10);
    }
    if (batch == 0) return TNG_OK;
    const uint64_t s = rows < cols ? rows : cols, l = rows < cols ? cols : rows;
    if (batch * up(l, 128) >= (1ull << 31) || (batch * up(s, 128) / 128) * (up(l, 128) / 128) >= (1ull << 31)) return TNG_ERR_INVALID_ARG;
    if (!matrix_ok(v_dev, type, cols, ldv) || !matrix_ok(out_dev, out_type, cols, ldo) || (batch > 1 && out_stride == 0) || !scratch_dev || !aligned(scratch_dev, 256)) return TNG_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    unsigned char* at = static_cast<unsigned char*>(scratch_dev);
    double* part = reinterpret_cast<double*>(at);
    Carver carve{at + batch * kNormBlocks * 8};
    const Halves x = carve.take(batch, s, l), g = carve.take(batch, s, s), poly = carve.take(batch, s, s);
    Halves xt = carve.take(batch, l, s), xt2 = carve.take(batch, l, s);
    const bool tall = rows > cols;
    cudaError_t e = with_type(type, [&](auto t) {
        using T = decltype(t);
        const T* v = static_cast<const T*>(v_dev);
        cudaError_t err = launch_layer(ortho_norm_kernel<T>, dim3(kNormBlocks, (unsigned)batch), 256, 0, 1, st, v, rows, cols, ldv, stride, part);
        if (err != cudaSuccess) return err;
        const dim3 grid((unsigned)((cols + 63) / 64), (unsigned)((rows + 63) / 64), (unsigned)batch);
        return launch_layer(ortho_split_kernel<T>, grid, 256, 0, 1, st, v, ldv, stride, static_cast<const double*>(part), tall ? xt : x, tall ? x : xt);
    });
    if (e != cudaSuccess) return layer_status(e);
    OrthoMaps gram = {}, square = {}, apply = {};
    bool made = make_maps(gram.p, x, batch, true) && make_maps(gram.d, g, batch, false) && make_maps(square.p, g, batch, true) &&
                make_maps(square.d, poly, batch, false) && make_maps(apply.d, x, batch, false);
    for (int i = 0; i < 2; ++i) {
        gram.q[i] = gram.p[i];
        gram.t[i] = gram.d[i];
        square.q[i] = square.p[i];
        square.t[i] = square.d[i];
    }
    OrthoMaps next = apply;
    made = made && make_maps(apply.p, poly, batch, true) && make_maps(apply.q, xt, batch, true) && make_maps(apply.t, xt2, batch, false) &&
           make_maps(next.q, xt2, batch, true) && make_maps(next.t, xt, batch, false);
    if (!made) return TNG_ERR_CUDA;
    next.p[0] = apply.p[0];
    next.p[1] = apply.p[1];
    OrthoArgs args = {};
    args.batch = (uint32_t)batch;
    for (uint32_t i = 0; i < steps; ++i) {
        const OrthoMaps& here = i & 1 ? next : apply;
        args.rows = args.cols = s;
        args.k = l;
        args.pad_p = args.pad_q = args.pad_d = args.pad_t = x.pad_rows;
        args.symmetric = 1;
        args.scale = kScaleG / (kScaleX * kScaleX);
        e = launch_product<kGram, float>(gram, args, st);
        if (e != cudaSuccess) return layer_status(e);
        args.k = s;
        args.g = g;
        args.scale = c * (kScaleB / (kScaleG * kScaleG));
        args.linear = b * (kScaleB / kScaleG);
        args.diagonal = a * kScaleB;
        e = launch_product<kPoly, float>(square, args, st);
        if (e != cudaSuccess) return layer_status(e);
        args.symmetric = 0;
        if (i + 1 < steps) {
            args.cols = l;
            args.pad_q = args.pad_t = xt.pad_rows;
            args.scale = kScaleX / (kScaleB * kScaleX);
            e = launch_product<kApply, float>(here, args, st);
        } else {
            // the last one as the output lies: B X, or X^T B
            OrthoMaps last = here;
            if (tall) {
                for (int j = 0; j < 2; ++j) {
                    last.p[j] = here.q[j];
                    last.q[j] = here.p[j];
                }
                args.pad_p = xt.pad_rows;
            } else {
                args.pad_q = xt.pad_rows;
            }
            args.rows = rows;
            args.cols = cols;
            args.scale = 1.f / (kScaleB * kScaleX);
            args.out = out_dev;
            args.ldo = ldo;
            args.stride = out_stride;
            e = with_type(out_type, [&](auto t) { return launch_product<kLast, decltype(t)>(last, args, st); });
        }
        if (e != cudaSuccess) return layer_status(e);
    }
    return TNG_OK;
}

}  // extern "C"
