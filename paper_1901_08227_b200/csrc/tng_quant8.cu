// 8-bit codes of a matrix with one scale a line: rows (a scale per token) or columns (a scale per
// channel, codes transposed).  The codes are unique: scale, 1/scale, product and (with a draw) the sum
// with the uniform are one fp32 rounding each, so any order of work gives the same bytes.
#include "tng_codes.cuh"

namespace tng {
namespace {

// ---- rows --------------------------------------------------------------------------------------------
// blockDim.x threads share a row, blockDim.y rows a CTA (more than one only where a row is one warp).
// Rows of up to 8 * kHold * blockDim.x columns are read once and kept in registers; longer ones twice.
constexpr int kHold = 4;
template <typename T, bool VEC, bool DRAW>
__global__ void quant8_rows_kernel(const T* __restrict__ x, uint64_t rows, uint64_t cols, uint64_t ldx, int8_t* __restrict__ q,
                                   uint64_t ldq, float* __restrict__ scale, const __grid_constant__ DrawArgs draw) {
    __shared__ uint32_t part[32];
    const uint64_t row = (uint64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= rows) return;                       // whole warps only: with blockDim.y > 1 there is no block barrier
    const T* src = x + row * ldx;
    const uint32_t groups = (uint32_t)((cols + 7) / 8), step = blockDim.x;
    float v[kHold][8];
    uint32_t m = 0;
#pragma unroll
    for (int h = 0; h < kHold; ++h) {
        const uint32_t g = threadIdx.x + h * step;
        if (g < groups) fetch8<T, VEC>(src, (uint64_t)g * 8, cols, v[h]);
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[h][j] = 0.f;
        }
    }
#pragma unroll
    for (int h = 0; h < kHold; ++h) m = max8(v[h], m);
    for (uint32_t g = threadIdx.x + kHold * step; g < groups; g += step) {
        float t[8];
        fetch8<T, VEC>(src, (uint64_t)g * 8, cols, t);
        m = max8(t, m);
    }
    m = __reduce_max_sync(kFullMask, m);
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
#pragma unroll
    for (int h = 0; h < kHold; ++h) {
        const uint32_t g = threadIdx.x + h * step;
        if (g < out_groups) dst[g] = g < groups ? code8<DRAW>(v[h], s.inv, draw, g, (uint32_t)row) : make_uint2(0u, 0u);
    }
    for (uint32_t g = threadIdx.x + kHold * step; g < out_groups; g += step) {
        float t[8] = {};
        if (g < groups) fetch8<T, VEC>(src, (uint64_t)g * 8, cols, t);
        dst[g] = g < groups ? code8<DRAW>(t, s.inv, draw, g, (uint32_t)row) : make_uint2(0u, 0u);
    }
}

// ---- columns -----------------------------------------------------------------------------------------
// Largest |x| and sum of every column over a chunk of rows.  A thread owns eight columns and every eighth row
// of the chunk; a CTA owns 256 columns.  Chunks are combined, in order, by the kernel that makes the codes.
constexpr int kStatCols = 256, kStatLanes = 8;
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) column_stats_kernel(const T* __restrict__ x, uint64_t rows, uint64_t cols, uint64_t ldx,
                                                           uint64_t rows_per_chunk, uint32_t* __restrict__ tops, float* __restrict__ sums) {
    __shared__ uint32_t sh_top[kStatLanes][kStatCols];
    __shared__ float sh_sum[kStatLanes][kStatCols];
    const uint32_t cg = threadIdx.x & 31, lane = threadIdx.x >> 5;
    const uint64_t c = (uint64_t)blockIdx.x * kStatCols + cg * 8;
    const uint64_t r0 = (uint64_t)blockIdx.y * rows_per_chunk;
    const uint64_t r1 = r0 + rows_per_chunk < rows ? r0 + rows_per_chunk : rows;
    uint32_t top[8] = {};
    float sum[8] = {};
    if (c < cols) {
#pragma unroll 4
        for (uint64_t r = r0 + lane; r < r1; r += kStatLanes) {
            float v[8];
            fetch8<T, VEC>(x + r * ldx, c, cols, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                top[j] = max(top[j], __float_as_uint(v[j]) & 0x7FFFFFFFu);
                sum[j] += v[j];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        sh_top[lane][cg * 8 + j] = top[j];
        sh_sum[lane][cg * 8 + j] = sum[j];
    }
    __syncthreads();
    const uint64_t col = (uint64_t)blockIdx.x * kStatCols + threadIdx.x;
    if (col >= cols) return;
    uint32_t t = 0;
    float s = 0.f;
#pragma unroll
    for (int l = 0; l < kStatLanes; ++l) {
        t = max(t, sh_top[l][threadIdx.x]);
        s += sh_sum[l][threadIdx.x];
    }
    tops[(uint64_t)blockIdx.y * cols + col] = t;
    if (sums) sums[(uint64_t)blockIdx.y * cols + col] = s;
}

// Codes, transposed.  A CTA owns 64 columns and kRowsPerCta rows, 128 rows at a time: a thread codes 4 rows x 8
// columns, packs the four rows of a column into a word (rows are contiguous in the output), and the words
// cross the CTA through shared memory so that a warp writes 128 contiguous bytes of one column.
constexpr int kColTile = 64, kRowTile = 128, kRowsPerCta = 512;
template <typename T, bool VEC, bool DRAW>
__global__ void __launch_bounds__(256) quant8_cols_kernel(const T* __restrict__ x, uint64_t rows, uint64_t cols, uint64_t ldx,
                                                          const uint32_t* __restrict__ tops, const float* __restrict__ sums, uint32_t chunks,
                                                          int8_t* __restrict__ q, uint64_t ldq, float* __restrict__ scale,
                                                          float* __restrict__ colsum, const __grid_constant__ DrawArgs draw) {
    __shared__ uint32_t words[kColTile][kRowTile / 4 + 1];
    __shared__ uint32_t sh_top[4][kColTile];
    __shared__ float sh_inv[kColTile];
    const uint32_t tiles = (uint32_t)((cols + kColTile - 1) / kColTile), slab = blockIdx.x / tiles;
    const uint64_t c0 = (uint64_t)(blockIdx.x - slab * tiles) * kColTile;
    {
        const uint32_t lc = threadIdx.x & 63, quarter = threadIdx.x >> 6;
        uint32_t t = 0;
        if (c0 + lc < cols)
            for (uint32_t k = quarter; k < chunks; k += 4) t = max(t, __ldg(tops + (uint64_t)k * cols + c0 + lc));
        sh_top[quarter][lc] = t;
        __syncthreads();
        if (threadIdx.x < kColTile) {
            t = max(max(sh_top[0][lc], sh_top[1][lc]), max(sh_top[2][lc], sh_top[3][lc]));
            const LineScale s = line_scale(t);
            sh_inv[lc] = s.inv;
            if (slab == 0 && c0 + lc < cols) {
                scale[c0 + lc] = s.scale;
                if (colsum) {
                    float a = 0.f;
                    for (uint32_t k = 0; k < chunks; ++k) a += __ldg(sums + (uint64_t)k * cols + c0 + lc);
                    colsum[c0 + lc] = a;
                }
            }
        }
        __syncthreads();
    }
    const uint32_t cg = threadIdx.x & 7, rg = threadIdx.x >> 3;       // eight columns, four rows
    const uint64_t c = c0 + cg * 8;
    float inv[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) inv[j] = sh_inv[cg * 8 + j];
    const uint64_t first = (uint64_t)slab * kRowsPerCta;
    const uint64_t last = first + kRowsPerCta < rows ? first + kRowsPerCta : rows;
    const uint64_t padded = (rows + 15) / 16 * 16;
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (uint64_t r0 = first; r0 < last; r0 += kRowTile) {
        uint32_t b[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t r = r0 + rg * 4 + i;
            float v[8] = {};
            if (r < rows && c < cols) fetch8<T, VEC>(x + r * ldx, c, cols, v);
            uint32_t w[8] = {};
            if constexpr (DRAW) {
                const uint4 wa = draw_words(draw, (uint32_t)(c >> 2), (uint32_t)r), wb = draw_words(draw, (uint32_t)(c >> 2) + 1, (uint32_t)r);
                w[0] = wa.x; w[1] = wa.y; w[2] = wa.z; w[3] = wa.w; w[4] = wb.x; w[5] = wb.y; w[6] = wb.z; w[7] = wb.w;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) b[i][j] = (r < rows && inv[j] != 0.f) ? code_bits<DRAW>(v[j], inv[j], w[j]) : 0u;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) words[cg * 8 + j][rg] = pack_bytes(b[0][j], b[1][j], b[2][j], b[3][j]);
        __syncthreads();
        const uint64_t r = r0 + lane * 4;
        if (r < padded) {
#pragma unroll
            for (int k = 0; k < kColTile / 8; ++k) {
                const uint32_t lc = warp + 8 * k;
                if (c0 + lc < cols) *reinterpret_cast<uint32_t*>(q + (c0 + lc) * ldq + r) = words[lc][lane];
            }
        }
        __syncthreads();
    }
}

uint32_t column_chunks(uint64_t rows, uint64_t cols) {
    const uint64_t blocks = (cols + kStatCols - 1) / kStatCols;
    uint64_t chunks = (148 * 4 + blocks - 1) / blocks;      // about four CTAs an SM
    const uint64_t most = (rows + 63) / 64;
    if (chunks > most) chunks = most;
    if (chunks > 64) chunks = 64;
    return chunks < 1 ? 1u : (uint32_t)chunks;
}

template <typename T, bool VEC, bool DRAW>
cudaError_t rows_launch(const void* x, uint64_t rows, uint64_t cols, uint64_t ldx, const DrawArgs& d, int8_t* q, uint64_t ldq,
                        float* scale, cudaStream_t st) {
    // a warp a row up to 1024 columns, eight rows a CTA; above, two groups of eight columns a thread
    const uint64_t groups = (cols + 7) / 8;
    dim3 block(32, 8);
    if (groups > 32 * kHold) {
        uint64_t t = (groups + 1) / 2;
        t = (t + 31) / 32 * 32;
        block = dim3((unsigned)(t > 512 ? 512 : t), 1);
    }
    const unsigned grid = (unsigned)((rows + block.y - 1) / block.y);
    quant8_rows_kernel<T, VEC, DRAW><<<grid, block, 0, st>>>(static_cast<const T*>(x), rows, cols, ldx, q, ldq, scale, d);
    return cudaGetLastError();
}

template <typename T, bool VEC>
cudaError_t cols_launch(const void* x, uint64_t rows, uint64_t cols, uint64_t ldx, const tng_draw* draw, int8_t* q, uint64_t ldq,
                        float* scale, float* colsum, void* scratch, cudaStream_t st) {
    const uint32_t chunks = column_chunks(rows, cols);
    uint32_t* tops = static_cast<uint32_t*>(scratch);
    float* sums = colsum ? reinterpret_cast<float*>(tops + (uint64_t)chunks * cols) : nullptr;
    const uint64_t per = (rows + chunks - 1) / chunks;
    const dim3 sg((unsigned)((cols + kStatCols - 1) / kStatCols), chunks);
    const T* px = static_cast<const T*>(x);
    column_stats_kernel<T, VEC><<<sg, 256, 0, st>>>(px, rows, cols, ldx, per, tops, sums);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    // one dimension, columns fastest: y would end at 65535 slabs, and neighbours share the rows' lines
    const uint64_t g = (cols + kColTile - 1) / kColTile * ((rows + kRowsPerCta - 1) / kRowsPerCta);
    if (g >= (1ull << 31)) return cudaErrorInvalidValue;
    if (draw) quant8_cols_kernel<T, VEC, true><<<(unsigned)g, 256, 0, st>>>(px, rows, cols, ldx, tops, sums, chunks, q, ldq, scale, colsum, make_draw(*draw, kTagRounding));
    else quant8_cols_kernel<T, VEC, false><<<(unsigned)g, 256, 0, st>>>(px, rows, cols, ldx, tops, sums, chunks, q, ldq, scale, colsum, DrawArgs{});
    return cudaGetLastError();
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
    return (size_t)(((uint64_t)column_chunks(rows, cols) * cols * 8 + 255) / 256 * 256);
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
