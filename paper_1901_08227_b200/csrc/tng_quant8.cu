// 8-bit codes of a matrix with one scale a line: rows (a scale per token) or columns (a scale per
// channel, codes transposed).  The codes are unique: scale, 1/scale, product and (with a draw) the sum
// with the uniform are one fp32 rounding each, so any order of work gives the same bytes.
#include "tng_codes.cuh"

namespace tng {
namespace {

// ---- rows --------------------------------------------------------------------------------------------
// blockDim.x threads share a row, blockDim.y rows a CTA (more than one only where a row is one warp).  A thread keeps
// up to 128 bytes of its row in registers as they came: all its loads are in flight at once, and the row is read once;
// longer rows (above 1024 threads' worth) are read twice.  16384 x 4096 bf16: 31 us, 6.4 TB/s; drawn 66 to 77 us, bound by
// issue slots (26 instructions an element and warp, 10 to nearest).
template <typename T> constexpr int kHold = 16 / (int)sizeof(T);       // groups of eight elements
template <typename T, bool VEC, bool DRAW>
__global__ void quant8_rows_kernel(const T* x, uint64_t rows, uint64_t cols, uint64_t ldx, int8_t* q,
                                   uint64_t ldq, float* scale, const __grid_constant__ DrawArgs draw) {
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
// Two passes, the first for the largest |x| and the sum of every column, the second for the codes; up to two matrices of
// one type a launch (a gradient's dy and x), of which the first may have its row codes made on the way (dy: one read
// less, and the random words of an element serve both its codes; the whole gradient at 2048 x 4096 x 4096, drawn: 102 -> 98 us).  (Panels of columns small enough for the L2 cache to hold between the passes
// saved the second read but lost as much to the ends of twice as many launches: 16384 x 4096 bf16, 83 us in panels of
// 64 MB, 76 us whole.)
template <typename T> struct ColumnJob {
    const T* x;
    uint64_t rows, cols, ldx, rows_per_chunk;
    uint32_t blocks, tiles, chunks;   // CTA columns of the first pass and of the second, row chunks of the first
    uint32_t per_cta;              // rows a CTA of the second pass: kRowsPerCta, or kRowTile where that leaves SMs idle
    uint32_t* tops;                // largest |x| as bit patterns, cleared before
    float* sums;                   // chunks x cols, or nullptr
    int8_t* q;
    uint64_t ldq;
    float *scale, *colsum;
    uint32_t* row_tops;            // with row codes too (else nullptr): largest |x| of the rows, cleared before
    int8_t* row_q;
    uint64_t ld_row;
    float* row_scale;
};
template <typename T> struct ColumnJobs {
    ColumnJob<T> job[2];
    uint32_t first2;               // first CTA of the second matrix
};

// Statistics.  A thread owns eight columns and every eighth row of a chunk; a CTA owns 256 columns.  Maxima meet in
// `tops` (cleared before) by atomic maximum of bit patterns, which no order changes; the chunks' sums are kept apart and
// added in order by the second pass.  16384 x 4096 bf16: 27 us cold, 5.2 TB/s.
constexpr int kStatCols = 256, kStatLanes = 8;
template <typename T, bool VEC>
__global__ void __launch_bounds__(256, 4) column_stats_kernel(const __grid_constant__ ColumnJobs<T> jobs) {
    constexpr int kWords = 2 * (int)sizeof(T);
    __shared__ uint32_t sh_top[kStatLanes][32 * kWords];
    __shared__ float sh_sum[kStatLanes][kStatCols];
    grid_wait();
    grid_go();
    const bool second = blockIdx.x >= jobs.first2;
    const ColumnJob<T>& job = jobs.job[second];
    const uint32_t cta = blockIdx.x - (second ? jobs.first2 : 0), chunk = cta / job.blocks;
    const uint64_t rows = job.rows, cols = job.cols, ldx = job.ldx;
    const T* x = job.x;
    const bool want_sums = job.sums != nullptr;
    const uint32_t cg = threadIdx.x & 31, lane = threadIdx.x >> 5;
    const uint64_t c0 = (uint64_t)(cta - chunk * job.blocks) * kStatCols, c = c0 + cg * 8;
    const uint64_t r0 = chunk * job.rows_per_chunk;
    const uint64_t r1 = r0 + job.rows_per_chunk < rows ? r0 + job.rows_per_chunk : rows;
    uint32_t top[kWords] = {};
    float sum[8] = {};
    const auto take = [&](const Raw8<T>& v, uint64_t r) {   // (columns past the end read as zero)
        const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
#pragma unroll
        for (int j = 0; j < kWords; ++j) top[j] = top_word<T>(w[j], top[j]);
        if (job.row_tops) {                                // a warp has 256 columns of one row
            const uint32_t m = __reduce_max_sync(kFullMask, top_of_halves<T>(top_raw8<T>(v, 0u)));
            if (cg == 0) atomicMax(job.row_tops + r, top_bits<T>(m));
        }
        if (want_sums) {
            float f[8];
            widen8(v, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += f[j];
        }
    };
    uint64_t r = r0 + lane;
    constexpr int kAhead = 8 / (int)sizeof(T);              // 64 bytes a thread in flight
    for (; r + (kAhead - 1) * kStatLanes < r1; r += kAhead * kStatLanes) {
        Raw8<T> v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) v[i] = fetch_raw8<T, VEC>(x + (r + i * kStatLanes) * ldx, c, cols);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) take(v[i], r + i * kStatLanes);
    }
    for (; r < r1; r += kStatLanes) take(fetch_raw8<T, VEC>(x + r * ldx, c, cols), r);
#pragma unroll
    for (int j = 0; j < kWords; ++j) sh_top[lane][cg * kWords + j] = top[j];
    if (want_sums) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sh_sum[lane][cg * 8 + j] = sum[j];
    }
    __syncthreads();
    const uint64_t col = c0 + threadIdx.x;
    if (col >= cols) return;
    constexpr int kPer = 4 / (int)sizeof(T);               // elements in a word
    uint32_t t = 0;
#pragma unroll
    for (int l = 0; l < kStatLanes; ++l) t = top_word<T>(sh_top[l][threadIdx.x / kPer], t);
    if (kPer == 2) t = threadIdx.x & 1 ? t >> 16 : t & 0xFFFFu;
    atomicMax(job.tops + col, top_bits<T>(t));
    if (want_sums) {
        float s = 0.f;
#pragma unroll
        for (int l = 0; l < kStatLanes; ++l) s += sh_sum[l][threadIdx.x];
        job.sums[(uint64_t)chunk * cols + col] = s;
    }
}

// Codes, transposed.  A CTA owns 64 columns and kRowsPerCta rows, 128 rows at a time: a thread codes 4 rows x 8
// columns, packs the four rows of a column into a word (rows are contiguous in the output), and the words
// cross the CTA through shared memory so that a warp writes 128 contiguous bytes of one column.  The next 128
// rows' loads are issued before that.  Both passes, 16384 x 4096 bf16: 60 to 64 us for 403 MB when the second read misses the
// L2 cache; drawn 100 to 104 us.
constexpr int kColTile = 64, kRowTile = 128, kRowsPerCta = 256;
template <typename T, bool VEC, bool DRAW, bool ROWS>
__global__ void __launch_bounds__(256, DRAW ? (ROWS ? 2 : 3) : (ROWS ? 3 : 4)) quant8_cols_kernel(const __grid_constant__ ColumnJobs<T> jobs, const __grid_constant__ DrawArgs draw) {
    __shared__ uint32_t words[2][kColTile][kRowTile / 4 + 1];
    __shared__ float sh_inv[kColTile], sh_sum[4][kColTile], sh_row_inv[ROWS ? kRowsPerCta : 1];
    grid_wait();
    grid_go();
    const bool second = blockIdx.x >= jobs.first2;
    const ColumnJob<T>& job = jobs.job[second];
    const uint32_t cta = blockIdx.x - (second ? jobs.first2 : 0), slab = cta / job.tiles;      // columns fastest: neighbours share the rows' lines
    const uint64_t rows = job.rows, cols = job.cols, ldx = job.ldx, ldq = job.ldq;
    const T* x = job.x;
    const uint64_t c0 = (uint64_t)(cta - slab * job.tiles) * kColTile;
    const uint32_t cg = threadIdx.x & 7, rg = threadIdx.x >> 3;       // eight columns, four rows
    const uint64_t c = c0 + cg * 8;
    const uint64_t first = (uint64_t)slab * job.per_cta;
    const uint64_t last = first + job.per_cta < rows ? first + job.per_cta : rows;
    const bool wide = VEC && c0 + kColTile <= cols;      // all 64 columns: vector loads, no tests on columns
    Raw8<T> v[4];
    const T* px = x + (first + rg * 4) * ldx + c;
    const auto fetch = [&](uint64_t r0) {                  // the next 128 rows, from r0
        if (wide && r0 + kRowTile <= last) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = load_raw8(px + i * ldx);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint64_t r = r0 + rg * 4 + i;
                v[i] = r < last && c < cols ? fetch_raw8<T, VEC>(x + r * ldx, c, cols) : zero_raw8<T>();
            }
        }
        px += kRowTile * ldx;
    };
    fetch(first);
    bool bad = false;                                      // a column with a NaN or infinity: rare, its codes are zero
    if (threadIdx.x < kColTile) {
        const uint64_t col = c0 + threadIdx.x;
        const uint32_t top = col < cols ? load4_bits(job.tops + col) : 0u;
        const LineScale s = line_scale(top);
        bad = top >= kInfBits;
        sh_inv[threadIdx.x] = s.inv;
        if (slab == 0 && col < cols) job.scale[col] = s.scale;
    }
    const bool rows_too = ROWS && job.row_q;
    if (rows_too) {
        static_assert(kRowsPerCta == 256, "a thread a row");
        const uint64_t r = first + threadIdx.x;
        const uint32_t top = r < last ? load4_bits(job.row_tops + r) : 0u;
        const LineScale s = line_scale(top);
        bad = bad || top >= kInfBits;
        sh_row_inv[threadIdx.x] = s.inv;
        if (c0 == 0 && r < last) job.row_scale[r] = s.scale;
    }
    if (slab == 0 && job.colsum) {                         // the chunks' sums: a quarter to a thread, the quarters in order
        const uint32_t lc = threadIdx.x & 63, quarter = threadIdx.x >> 6;
        float a = 0.f;
        if (c0 + lc < cols) {                              // eight loads under way at a time
            const uint32_t k0 = job.chunks * quarter / 4, k1 = job.chunks * (quarter + 1) / 4;
            for (uint32_t k = k0; k < k1; k += 8) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = load_f32(job.sums + (uint64_t)(k + i < k1 ? k + i : k1 - 1) * cols + c0 + lc);
#pragma unroll
                for (int i = 0; i < 8; ++i) a += k + i < k1 ? v[i] : 0.f;
            }
        }
        sh_sum[quarter][lc] = a;
    }
    const bool any_bad = __syncthreads_or(bad);
    if (slab == 0 && job.colsum && threadIdx.x < kColTile && c0 + threadIdx.x < cols)
        job.colsum[c0 + threadIdx.x] = (sh_sum[0][threadIdx.x] + sh_sum[1][threadIdx.x]) + (sh_sum[2][threadIdx.x] + sh_sum[3][threadIdx.x]);
    float inv[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) inv[j] = sh_inv[cg * 8 + j];
    const uint64_t padded = (rows + 15) / 16 * 16, column = draw_column((uint32_t)(c >> 2));
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int8_t* dst = job.q + (c0 + warp) * ldq + first + lane * 4;
    uint32_t flip = 0;
    for (uint64_t r0 = first; r0 < last; r0 += kRowTile, flip ^= 1) {
        uint32_t pairs[8];                                 // codes of rows 0 and 1 in the low bytes, then all four
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t b[2][8];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float f[8];
                widen8(v[2 * h + i], f);
                uint32_t w[8] = {};
                if constexpr (DRAW) {
                    const DrawRow dr = draw_row(draw, (uint32_t)r0 + rg * 4 + 2 * h + i);
                    const uint4 wa = draw_words(draw, dr, column), wb = draw_words(draw, dr, column + kPhiloxMul0);
                    w[0] = wa.x; w[1] = wa.y; w[2] = wa.z; w[3] = wa.w; w[4] = wb.x; w[5] = wb.y; w[6] = wb.z; w[7] = wb.w;
                }
                // (rows past the end read as zero, a zero column has inv = 0: code zero, with a draw too, since floor(0 + u) = 0)
#pragma unroll
                for (int j = 0; j < 8; ++j) b[i][j] = code_bits<DRAW>(f[j], inv[j], w[j]);
                if (rows_too) {
                    const uint32_t at = rg * 4 + 2 * h + i;            // of these 128 rows
                    const uint64_t r = r0 + at;
                    const float inv_r = sh_row_inv[(uint32_t)(r0 - first) + at];
                    uint32_t e[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) e[j] = code_bits<DRAW>(f[j], inv_r, w[j]);
                    uint2 out = make_uint2(pack_bytes(e[0], e[1], e[2], e[3]), pack_bytes(e[4], e[5], e[6], e[7]));
                    if (any_bad && inv_r == 0.f) out = make_uint2(0u, 0u);
                    // (zeros up to the next multiple of 16, like the columns past the end that they are)
                    if (r < last && (wide || c < (cols + 15) / 16 * 16)) *reinterpret_cast<uint2*>(job.row_q + r * job.ld_row + c) = out;
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t two = __byte_perm(b[0][j], b[1][j], 0x0040);
                pairs[j] = h ? __byte_perm(pairs[j], two, 0x5410) : two;
            }
        }
        if (any_bad) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (inv[j] == 0.f) pairs[j] = 0u;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) words[flip][cg * 8 + j][rg] = pairs[j];
        __syncthreads();                                   // (the half written next was read before this barrier)
        if (r0 + kRowTile < last) fetch(r0 + kRowTile);
        if (r0 + lane * 4 < padded) {
            int8_t* to = dst;
#pragma unroll
            for (int k = 0; k < kColTile / 8; ++k, to += 8 * ldq) {
                const uint32_t lc = warp + 8 * k;
                if (wide || c0 + lc < cols) *reinterpret_cast<uint32_t*>(to) = words[flip][lc][lane];
            }
        }
        dst += kRowTile;
    }
}

// Row chunks of the statistics: about four CTAs an SM, and a chunk for every 32 rows at most (33 rows are two of 17 and 16).  The
// SMs are a B200's, not those of the current device: the sizes of scratch follow from the chunks.
constexpr uint64_t kStatCtas = 4 * 148;
uint32_t column_chunks(uint64_t rows, uint64_t cols) {
    const uint64_t blocks = (cols + kStatCols - 1) / kStatCols;
    uint64_t chunks = (kStatCtas + blocks - 1) / blocks;
    const uint64_t most = (rows + 31) / 32;
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

template <typename T, bool VEC, bool ROWS>
cudaError_t cols_launch(const ColumnJobs<T>& jobs, const DrawArgs* draw, uint64_t ctas1, uint64_t ctas2, cudaStream_t st) {
    ColumnJobs<T> j = jobs;
    j.first2 = (uint32_t)((uint64_t)j.job[0].blocks * j.job[0].chunks);
    cudaError_t e = launch_layer(column_stats_kernel<T, VEC>, j.first2 + j.job[1].blocks * j.job[1].chunks, 256, 0, 1, st, j);
    if (e != cudaSuccess) return e;
    j.first2 = (uint32_t)ctas1;
    return draw ? launch_layer(quant8_cols_kernel<T, VEC, true, ROWS>, (unsigned)(ctas1 + ctas2), 256, 0, 1, st, j, *draw)
                : launch_layer(quant8_cols_kernel<T, VEC, false, ROWS>, (unsigned)(ctas1 + ctas2), 256, 0, 1, st, j, DrawArgs{});
}

template <typename T> bool rows_aligned(const void* x, uint64_t rows, uint64_t ldx) {
    return aligned(x, 16) && (rows == 1 || ldx * sizeof(T) % 16 == 0);
}

}  // namespace

cudaError_t launch_quant8_rows(const void* x, tng_dtype type, uint64_t rows, uint64_t cols, uint64_t ldx, const tng_draw* draw,
                               int8_t* q, uint64_t ldq, float* scale, cudaStream_t st) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        const DrawArgs d = draw ? make_draw(*draw, kTagRounding) : DrawArgs{};
        const auto launch = rows_aligned<T>(x, rows, ldx) ? (draw ? rows_launch<T, true, true> : rows_launch<T, true, false>)
                                                          : (draw ? rows_launch<T, false, true> : rows_launch<T, false, false>);
        return launch(x, rows, cols, ldx, d, q, ldq, scale, st);
    });
}

uint64_t quant8_cols_scratch(uint64_t rows, uint64_t cols) { return (1 + (uint64_t)column_chunks(rows, cols)) * cols; }

// Jobs of one type whose maxima (the first words of their scratch, row_tops) are clear; only the first may have row codes.  Two of them share the launches where
// they are alike in alignment and neither is drawn.
cudaError_t launch_quant8_cols(const Quant8Cols* jobs, int n, tng_dtype type, cudaStream_t st) {
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        ColumnJobs<T> j = {};
        uint64_t ctas[2] = {};
        bool vec[2] = {};
        for (int i = 0; i < n; ++i) {
            const Quant8Cols& in = jobs[i];
            ColumnJob<T>& o = j.job[i];
            o.x = static_cast<const T*>(in.x);
            o.rows = in.rows; o.cols = in.cols; o.ldx = in.ldx;
            o.chunks = column_chunks(in.rows, in.cols);
            o.rows_per_chunk = (in.rows + o.chunks - 1) / o.chunks;
            o.blocks = (uint32_t)((in.cols + kStatCols - 1) / kStatCols);
            o.tiles = (uint32_t)((in.cols + kColTile - 1) / kColTile);
            o.tops = in.scratch;
            o.sums = in.colsum ? reinterpret_cast<float*>(in.scratch + in.cols) : nullptr;
            o.q = in.q; o.ldq = in.ldq; o.scale = in.scale; o.colsum = in.colsum;
            o.row_tops = in.row_tops; o.row_q = in.row_q; o.ld_row = in.ld_row; o.row_scale = in.row_scale;
            ctas[i] = o.tiles * ((in.rows + kRowsPerCta - 1) / kRowsPerCta);
            o.per_cta = ctas[i] < 2ull * sm_count_now() ? kRowTile : kRowsPerCta;
            ctas[i] = o.tiles * ((in.rows + o.per_cta - 1) / o.per_cta);
            vec[i] = rows_aligned<T>(in.x, in.rows, in.ldx);
        }
        if (ctas[0] + ctas[1] >= (1ull << 31)) return cudaErrorInvalidValue;
        const auto one = [&](const ColumnJobs<T>& k, const tng_draw* draw, bool v, uint64_t c1, uint64_t c2) {
            const DrawArgs d = draw ? make_draw(*draw, kTagRounding) : DrawArgs{};
            const auto launch = k.job[0].row_q ? (v ? cols_launch<T, true, true> : cols_launch<T, false, true>)
                                               : (v ? cols_launch<T, true, false> : cols_launch<T, false, false>);
            return launch(k, draw ? &d : nullptr, c1, c2, st);
        };
        if (n == 1) return one(j, jobs[0].draw, vec[0], ctas[0], 0);
        if (vec[0] == vec[1] && !jobs[0].draw && !jobs[1].draw) return one(j, nullptr, vec[0], ctas[0], ctas[1]);
        for (int i = 0; i < 2; ++i) {
            ColumnJobs<T> k = {};
            k.job[0] = j.job[i];
            const cudaError_t e = one(k, jobs[i].draw, vec[i], ctas[i], 0);
            if (e != cudaSuccess) return e;
        }
        return cudaSuccess;
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
    return layer_status(launch_quant8_rows(x_dev, type, rows, cols, ldx, draw, q_dev, ldq, scale_dev, static_cast<cudaStream_t>(stream)));
}

size_t tng_quant8_cols_scratch_bytes(uint64_t rows, uint64_t cols) {
    return (size_t)((quant8_cols_scratch(rows, cols) * 4 + 255) / 256 * 256);
}

tng_status tng_quant8_cols(const void* x_dev, tng_dtype type, uint64_t rows, uint64_t cols, uint64_t ldx, const tng_draw* draw,
                           int8_t* q_dev, uint64_t ldq, float* scale_dev, float* colsum_dev, void* scratch_dev, void* stream) {
    if (!type_ok(type) || cols < 1 || !dims_ok(rows, cols) || (draw && !draw_ok(draw, rows))) return TNG_ERR_INVALID_ARG;
    if (!scale_dev || !aligned(scale_dev, 4) || !aligned(colsum_dev, 4)) return TNG_ERR_INVALID_ARG;
    if (rows == 0) {                               // columns of nothing: scale and sum zero
        cudaStream_t st = static_cast<cudaStream_t>(stream);
        cudaError_t e = cudaMemsetAsync(scale_dev, 0, cols * 4, st);
        if (e == cudaSuccess && colsum_dev) e = cudaMemsetAsync(colsum_dev, 0, cols * 4, st);
        return layer_status(e);
    }
    if (!matrix_ok(x_dev, type, cols, ldx) || !codes_ok(q_dev, rows, ldq) || !scratch_dev || !aligned(scratch_dev, 256))
        return TNG_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint32_t* scratch = static_cast<uint32_t*>(scratch_dev);
    const cudaError_t e = cudaMemsetAsync(scratch, 0, cols * 4, st);
    if (e != cudaSuccess) return layer_status(e);
    const Quant8Cols job{x_dev, rows, cols, ldx, draw, q_dev, ldq, scale_dev, colsum_dev, scratch, nullptr, nullptr, 0, nullptr};
    return layer_status(launch_quant8_cols(&job, 1, type, st));
}

}  // extern "C"
