// 8-bit codes of a matrix with one scale a line: rows (a scale per token) or columns (a scale per
// channel, codes transposed).  The codes are unique: scale, 1/scale, product and (with a draw) the sum
// with the uniform are one fp32 rounding each, so any order of work gives the same bytes.
#include "tng_codes.cuh"

namespace tng {
namespace {

// ---- rows --------------------------------------------------------------------------------------------
// blockDim.x threads share a row, blockDim.y rows a CTA (more than one only where a row is one warp).  A thread keeps
// up to 128 bytes of its row in registers as they came: all its loads are in flight at once, and the row is read once;
// longer rows (above 1024 threads' worth) are read twice.
template <typename T> constexpr int kHold = 16 / (int)sizeof(T);       // groups of eight elements
template <typename T, bool VEC, bool DRAW>
__global__ void quant8_rows_kernel(const T* __restrict__ x, uint64_t rows, uint64_t cols, uint64_t ldx, int8_t* __restrict__ q,
                                   uint64_t ldq, float* __restrict__ scale, const __grid_constant__ DrawArgs draw) {
    __shared__ uint32_t part[32];
    grid_wait();
    grid_go();
    const uint64_t row = (uint64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= rows) return;                       // whole warps only: with blockDim.y > 1 there is no block barrier
    const T* src = x + row * ldx;
    const uint32_t groups = (uint32_t)((cols + 7) / 8), step = blockDim.x;
    Raw8<T> v[kHold<T>];
    uint32_t m = 0;
#pragma unroll
    for (int h = 0; h < kHold<T>; ++h) {
        const uint32_t g = threadIdx.x + h * step;
        v[h] = g < groups ? fetch_raw8<T, VEC>(src, (uint64_t)g * 8, cols) : zero_raw8<T>();
    }
#pragma unroll
    for (int h = 0; h < kHold<T>; ++h) m = top_raw8<T>(v[h], m);
    for (uint32_t g = threadIdx.x + kHold<T> * step; g < groups; g += step) m = top_raw8<T>(fetch_raw8<T, VEC>(src, (uint64_t)g * 8, cols), m);
    m = __reduce_max_sync(kFullMask, top_bits<T>(top_of_halves<T>(m)));
    if (blockDim.x > 32) {
        const uint32_t lane = threadIdx.x & 31, warps = blockDim.x >> 5;
        if (lane == 0) part[threadIdx.x >> 5] = m;
        __syncthreads();
        m = __reduce_max_sync(kFullMask, lane < warps ? part[lane] : 0u);
    }
    const LineScale s = line_scale(m);
    if (threadIdx.x == 0) scale[row] = s.scale;
    const uint32_t out_groups = (uint32_t)((cols + 15) / 16 * 2);      // zeros up to the next multiple of 16
    uint2* dst = reinterpret_cast<uint2*>(q + row * ldq);
    DrawRow dr = {};
    if constexpr (DRAW) dr = draw_row(draw, (uint32_t)row);
    const auto put = [&](uint32_t g, const Raw8<T>& r) {
        float f[8];
        widen8(r, f);
        dst[g] = g < groups ? code8<DRAW>(f, s.inv, draw, dr, g) : make_uint2(0u, 0u);
    };
#pragma unroll
    for (int h = 0; h < kHold<T>; ++h) {
        const uint32_t g = threadIdx.x + h * step;
        if (g < out_groups) put(g, v[h]);
    }
    for (uint32_t g = threadIdx.x + kHold<T> * step; g < out_groups; g += step)
        put(g, g < groups ? fetch_raw8<T, VEC>(src, (uint64_t)g * 8, cols) : zero_raw8<T>());
}

// ---- columns -----------------------------------------------------------------------------------------
// Two passes over a panel of columns that the L2 cache can hold, so that the second finds the panel there: largest |x|
// and sum of every column, then the codes.
//
// Statistics.  A thread owns eight columns and every eighth row of a chunk; a CTA owns 256 columns.  Maxima meet in
// `tops` (cleared before) by atomic maximum of bit patterns, which no order changes; the chunks' sums are kept apart and
// added in order by the second pass.
constexpr int kStatCols = 256, kStatLanes = 8;
template <typename T, bool VEC, bool SUMS>
__global__ void __launch_bounds__(256, 4) column_stats_kernel(const T* __restrict__ x, uint64_t rows, uint64_t cols, uint64_t ldx, uint64_t c_first,
                                                           uint64_t c_last, uint64_t rows_per_chunk, uint32_t* __restrict__ tops,
                                                           float* __restrict__ sums) {
    constexpr int kWords = 2 * (int)sizeof(T);
    __shared__ uint32_t sh_top[kStatLanes][32 * kWords];
    __shared__ float sh_sum[SUMS ? kStatLanes : 1][kStatCols];
    grid_wait();
    grid_go();
    const uint32_t cg = threadIdx.x & 31, lane = threadIdx.x >> 5;
    const uint64_t c0 = c_first + (uint64_t)blockIdx.x * kStatCols, c = c0 + cg * 8;
    const uint64_t r0 = (uint64_t)blockIdx.y * rows_per_chunk;
    const uint64_t r1 = r0 + rows_per_chunk < rows ? r0 + rows_per_chunk : rows;
    uint32_t top[kWords] = {};
    float sum[8] = {};
    if (c < c_last) {
        const auto take = [&](const Raw8<T>& r) {
            const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
            for (int j = 0; j < kWords; ++j) top[j] = top_word<T>(w[j], top[j]);
            if (SUMS) {
                float v[8];
                widen8(r, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += v[j];
            }
        };
        uint64_t r = r0 + lane;
        constexpr int kAhead = 8 / (int)sizeof(T);          // 64 bytes a thread in flight
        for (; r + (kAhead - 1) * kStatLanes < r1; r += kAhead * kStatLanes) {
            Raw8<T> v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) v[i] = fetch_raw8<T, VEC>(x + (r + i * kStatLanes) * ldx, c, cols);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) take(v[i]);
        }
        for (; r < r1; r += kStatLanes) take(fetch_raw8<T, VEC>(x + r * ldx, c, cols));
    }
#pragma unroll
    for (int j = 0; j < kWords; ++j) sh_top[lane][cg * kWords + j] = top[j];
    if (SUMS) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sh_sum[lane][cg * 8 + j] = sum[j];
    }
    __syncthreads();
    const uint64_t col = c0 + threadIdx.x;
    if (col >= c_last) return;
    constexpr int kPer = 4 / (int)sizeof(T);               // elements in a word
    uint32_t t = 0;
#pragma unroll
    for (int l = 0; l < kStatLanes; ++l) t = top_word<T>(sh_top[l][threadIdx.x / kPer], t);
    if (kPer == 2) t = threadIdx.x & 1 ? t >> 16 : t & 0xFFFFu;
    atomicMax(tops + col, top_bits<T>(t));
    if (SUMS) {
        float s = 0.f;
#pragma unroll
        for (int l = 0; l < kStatLanes; ++l) s += sh_sum[l][threadIdx.x];
        sums[(uint64_t)blockIdx.y * cols + col] = s;
    }
}

// Codes, transposed.  A CTA owns 64 columns and kRowsPerCta rows, 128 rows at a time: a thread codes 4 rows x 8
// columns, packs the four rows of a column into a word (rows are contiguous in the output), and the words
// cross the CTA through shared memory so that a warp writes 128 contiguous bytes of one column.  The next 128
// rows' loads are issued before that.
constexpr int kColTile = 64, kRowTile = 128, kRowsPerCta = 512;
template <typename T, bool VEC, bool DRAW>
__global__ void __launch_bounds__(256, DRAW ? 3 : 4) quant8_cols_kernel(const T* __restrict__ x, uint64_t rows, uint64_t cols, uint64_t ldx, uint64_t c_first,
                                                          uint64_t c_last, const uint32_t* __restrict__ tops, const float* __restrict__ sums,
                                                          uint32_t chunks, int8_t* __restrict__ q, uint64_t ldq, float* __restrict__ scale,
                                                          float* __restrict__ colsum, const __grid_constant__ DrawArgs draw) {
    __shared__ uint32_t words[kColTile][kRowTile / 4 + 1];
    __shared__ float sh_inv[kColTile], sh_sum[4][kColTile];
    grid_wait();
    grid_go();
    const uint32_t tiles = (uint32_t)((c_last - c_first + kColTile - 1) / kColTile), slab = blockIdx.x / tiles;
    const uint64_t c0 = c_first + (uint64_t)(blockIdx.x - slab * tiles) * kColTile;
    const uint32_t cg = threadIdx.x & 7, rg = threadIdx.x >> 3;       // eight columns, four rows
    const uint64_t c = c0 + cg * 8;
    const uint64_t first = (uint64_t)slab * kRowsPerCta;
    const uint64_t last = first + kRowsPerCta < rows ? first + kRowsPerCta : rows;
    Raw8<T> v[4];
    const auto fetch = [&](uint64_t r0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t r = r0 + rg * 4 + i;
            v[i] = r < last && c < c_last ? fetch_raw8<T, VEC>(x + r * ldx, c, cols) : zero_raw8<T>();
        }
    };
    fetch(first);
    if (threadIdx.x < kColTile) {
        const uint64_t col = c0 + threadIdx.x;
        const LineScale s = line_scale(col < c_last ? __ldg(tops + col) : 0u);
        sh_inv[threadIdx.x] = s.inv;
        if (slab == 0 && col < c_last) scale[col] = s.scale;
    }
    if (slab == 0 && colsum) {                             // the chunks' sums: a quarter to a thread, the quarters in order
        const uint32_t lc = threadIdx.x & 63, quarter = threadIdx.x >> 6;
        float a = 0.f;
        if (c0 + lc < c_last) {
#pragma unroll 8
            for (uint32_t k = chunks * quarter / 4; k < chunks * (quarter + 1) / 4; ++k) a += __ldg(sums + (uint64_t)k * cols + c0 + lc);
        }
        sh_sum[quarter][lc] = a;
    }
    __syncthreads();
    if (slab == 0 && colsum && threadIdx.x < kColTile && c0 + threadIdx.x < c_last)
        colsum[c0 + threadIdx.x] = (sh_sum[0][threadIdx.x] + sh_sum[1][threadIdx.x]) + (sh_sum[2][threadIdx.x] + sh_sum[3][threadIdx.x]);
    float inv[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) inv[j] = sh_inv[cg * 8 + j];
    const uint64_t padded = (rows + 15) / 16 * 16, column = draw_column((uint32_t)(c >> 2));
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (uint64_t r0 = first; r0 < last; r0 += kRowTile) {
        uint32_t b[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t r = r0 + rg * 4 + i;
            float f[8];
            widen8(v[i], f);
            uint32_t w[8] = {};
            if constexpr (DRAW) {
                const DrawRow dr = draw_row(draw, (uint32_t)r);
                const uint4 wa = draw_words(draw, dr, column), wb = draw_words(draw, dr, column + kPhiloxMul0);
                w[0] = wa.x; w[1] = wa.y; w[2] = wa.z; w[3] = wa.w; w[4] = wb.x; w[5] = wb.y; w[6] = wb.z; w[7] = wb.w;
            }
            // (a column that is zero or not finite has inv = 0: code zero also where 0 * x is NaN; rows past the end read as
            // zero, and floor(0 + u) = 0)
#pragma unroll
            for (int j = 0; j < 8; ++j) b[i][j] = inv[j] != 0.f ? code_bits<DRAW>(f[j], inv[j], w[j]) : 0u;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) words[cg * 8 + j][rg] = pack_bytes(b[0][j], b[1][j], b[2][j], b[3][j]);
        __syncthreads();
        if (r0 + kRowTile < last) fetch(r0 + kRowTile);
        const uint64_t r = r0 + lane * 4;
        if (r < padded) {
#pragma unroll
            for (int k = 0; k < kColTile / 8; ++k) {
                const uint32_t lc = warp + 8 * k;
                if (c0 + lc < c_last) *reinterpret_cast<uint32_t*>(q + (c0 + lc) * ldq + r) = words[lc][lane];
            }
        }
        __syncthreads();
    }
}

// Columns of a panel: what 32 MB hold, in whole CTAs.
uint64_t panel_columns(uint64_t rows, uint64_t cols, uint64_t element) {
    uint64_t n = (32ull << 20) / (rows * element) / kStatCols * kStatCols;
    if (n < kStatCols) n = kStatCols;
    return n < cols ? n : cols;
}
// Row chunks of the statistics: about four CTAs an SM, 64 rows at least.
uint32_t column_chunks(uint64_t rows, uint64_t panel) {
    const uint64_t blocks = (panel + kStatCols - 1) / kStatCols;
    uint64_t chunks = (4 * 148 + blocks - 1) / blocks;
    const uint64_t most = (rows + 63) / 64;
    if (chunks > most) chunks = most;
    return chunks < 1 ? 1u : (uint32_t)chunks;
}

template <typename T, bool VEC, bool DRAW>
cudaError_t rows_launch(const void* x, uint64_t rows, uint64_t cols, uint64_t ldx, const DrawArgs& d, int8_t* q, uint64_t ldq,
                        float* scale, cudaStream_t st) {
    // a warp a row while it can hold one, eight rows a CTA; above, as many threads as hold the row
    const uint64_t groups = (cols + 7) / 8;
    dim3 block(32, 8);
    if (groups > 32 * kHold<T>) {
        const uint64_t t = (groups + 32 * kHold<T> - 1) / (32 * kHold<T>) * 32;
        block = dim3((unsigned)(t > 1024 ? 1024 : t), 1);
    }
    const unsigned grid = (unsigned)((rows + block.y - 1) / block.y);
    return launch_layer(quant8_rows_kernel<T, VEC, DRAW>, grid, block, 0, 1, st, static_cast<const T*>(x), rows, cols, ldx, q, ldq, scale, d);
}

template <typename T, bool VEC>
cudaError_t cols_launch(const void* x, uint64_t rows, uint64_t cols, uint64_t ldx, const tng_draw* draw, int8_t* q, uint64_t ldq,
                        float* scale, float* colsum, void* scratch, cudaStream_t st) {
    uint32_t* tops = static_cast<uint32_t*>(scratch);
    float* sums = reinterpret_cast<float*>(tops + cols);
    const T* px = static_cast<const T*>(x);
    const uint64_t panel = panel_columns(rows, cols, sizeof(T));
    const uint32_t chunks = column_chunks(rows, panel);
    const uint64_t per = (rows + chunks - 1) / chunks, slabs = (rows + kRowsPerCta - 1) / kRowsPerCta;
    if ((panel + kColTile - 1) / kColTile * slabs >= (1ull << 31)) return cudaErrorInvalidValue;
    cudaError_t e = cudaMemsetAsync(tops, 0, cols * 4, st);
    const DrawArgs d = draw ? make_draw(*draw, kTagRounding) : DrawArgs{};
    for (uint64_t c0 = 0; c0 < cols && e == cudaSuccess; c0 += panel) {
        const uint64_t c1 = c0 + panel < cols ? c0 + panel : cols;
        const dim3 sg((unsigned)((c1 - c0 + kStatCols - 1) / kStatCols), chunks);
        e = colsum ? launch_layer(column_stats_kernel<T, VEC, true>, sg, 256, 0, 1, st, px, rows, cols, ldx, c0, c1, per, tops, sums)
                   : launch_layer(column_stats_kernel<T, VEC, false>, sg, 256, 0, 1, st, px, rows, cols, ldx, c0, c1, per, tops, sums);
        if (e != cudaSuccess) break;
        // one dimension, columns fastest: neighbours share the rows' lines
        const unsigned g = (unsigned)((c1 - c0 + kColTile - 1) / kColTile * slabs);
        e = draw ? launch_layer(quant8_cols_kernel<T, VEC, true>, g, 256, 0, 1, st, px, rows, cols, ldx, c0, c1, tops, sums, chunks, q, ldq, scale, colsum, d)
                 : launch_layer(quant8_cols_kernel<T, VEC, false>, g, 256, 0, 1, st, px, rows, cols, ldx, c0, c1, tops, sums, chunks, q, ldq, scale, colsum, d);
    }
    return e;
}

template <typename T> bool rows_aligned(const void* x, uint64_t rows, uint64_t ldx) {
    return aligned(x, 16) && (rows == 1 || ldx * sizeof(T) % 16 == 0);
}

}  // namespace

cudaError_t launch_quant8_rows(const void* x, tng_dtype type, uint64_t rows, uint64_t cols, uint64_t ldx, const tng_draw* draw,
                               int8_t* q, uint64_t ldq, float* scale, cudaStream_t st) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        const bool vec = rows_aligned<T>(x, rows, ldx);
        const DrawArgs d = draw ? make_draw(*draw, kTagRounding) : DrawArgs{};
        if (vec) return draw ? rows_launch<T, true, true>(x, rows, cols, ldx, d, q, ldq, scale, st) : rows_launch<T, true, false>(x, rows, cols, ldx, d, q, ldq, scale, st);
        return draw ? rows_launch<T, false, true>(x, rows, cols, ldx, d, q, ldq, scale, st) : rows_launch<T, false, false>(x, rows, cols, ldx, d, q, ldq, scale, st);
    });
}

cudaError_t launch_quant8_cols(const void* x, tng_dtype type, uint64_t rows, uint64_t cols, uint64_t ldx, const tng_draw* draw,
                               int8_t* q, uint64_t ldq, float* scale, float* colsum, void* scratch, cudaStream_t st) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        return rows_aligned<T>(x, rows, ldx) ? cols_launch<T, true>(x, rows, cols, ldx, draw, q, ldq, scale, colsum, scratch, st)
                                             : cols_launch<T, false>(x, rows, cols, ldx, draw, q, ldq, scale, colsum, scratch, st);
    });
}

}  // namespace tng

using namespace tng;

extern "C" {

size_t tng_code_stride(uint64_t n) { return (size_t)((n + 15) / 16 * 16); }

tng_status tng_quant8_rows(const void* x_dev, tng_dtype type, uint64_t rows, uint64_t cols, uint64_t ldx, const tng_draw* draw,
                           int8_t* q_dev, uint64_t ldq, float* scale_dev, void* stream) {
    if (!type_ok(type) || cols < 1 || !dims_ok(rows, cols) || (draw && !draw_ok(draw, rows))) return TNG_ERR_INVALID_ARG;
    if (rows == 0) return TNG_OK;
    if (!matrix_ok(x_dev, type, cols, ldx) || !codes_ok(q_dev, cols, ldq) || !scale_dev || !aligned(scale_dev, 4)) return TNG_ERR_INVALID_ARG;
    return launch_quant8_rows(x_dev, type, rows, cols, ldx, draw, q_dev, ldq, scale_dev, static_cast<cudaStream_t>(stream)) == cudaSuccess
               ? TNG_OK : TNG_ERR_CUDA;
}

size_t tng_quant8_cols_scratch_bytes(uint64_t rows, uint64_t cols) {
    // maxima and the chunks' sums; chunks for the narrowest panel that any element type gives
    const uint64_t panel = rows ? panel_columns(rows, cols, 4) : 1;
    return (size_t)(((1 + (uint64_t)column_chunks(rows, panel)) * cols * 4 + 255) / 256 * 256);
}

tng_status tng_quant8_cols(const void* x_dev, tng_dtype type, uint64_t rows, uint64_t cols, uint64_t ldx, const tng_draw* draw,
                           int8_t* q_dev, uint64_t ldq, float* scale_dev, float* colsum_dev, void* scratch_dev, void* stream) {
    if (!type_ok(type) || cols < 1 || !dims_ok(rows, cols) || (draw && !draw_ok(draw, rows))) return TNG_ERR_INVALID_ARG;
    if (!scale_dev || !aligned(scale_dev, 4) || !aligned(colsum_dev, 4)) return TNG_ERR_INVALID_ARG;
    if (rows == 0) {                               // columns of nothing: scale and sum zero
        cudaStream_t st = static_cast<cudaStream_t>(stream);
        if (cudaMemsetAsync(scale_dev, 0, cols * 4, st) != cudaSuccess) return TNG_ERR_CUDA;
        return !colsum_dev || cudaMemsetAsync(colsum_dev, 0, cols * 4, st) == cudaSuccess ? TNG_OK : TNG_ERR_CUDA;
    }
    if (!matrix_ok(x_dev, type, cols, ldx) || !codes_ok(q_dev, rows, ldq) || !scratch_dev || !aligned(scratch_dev, 256))
        return TNG_ERR_INVALID_ARG;
    return launch_quant8_cols(x_dev, type, rows, cols, ldx, draw, q_dev, ldq, scale_dev, colsum_dev, scratch_dev,
                              static_cast<cudaStream_t>(stream)) == cudaSuccess ? TNG_OK : TNG_ERR_CUDA;
}

}  // extern "C"
