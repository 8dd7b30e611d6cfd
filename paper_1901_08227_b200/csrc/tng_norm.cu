// Root-mean-square norm with the residual's addition, its output in 8 bits with a scale a row or in the rows' own type, and its
// gradient.
//
//   h = x + residual (rounded to the type), r = 1 / sqrt(mean(h^2) + eps), y = h r w
//   codes of y by row: with t = h w and A = max|t|, q = rint(t 127/A), scale = (A/127) r
//
// r is the same for a whole row, so it cancels in the codes: they follow from h and w by one fp32 product, one quotient and one
// more product, whatever the order in which the squares are added, and every variant below gives the same bytes.  It also
// lets the sum of squares and the maximum be formed together, in one pass and one meeting of the row's threads.
//
// Both directions are bound by memory.  A thread owns the same columns of every row it works on: the weights (and in the
// gradient their sums) stay in its registers.
#include "tng_codes.cuh"

namespace tng {
namespace {

struct NormArgs {
    const void *x, *residual;
    const float* w;
    void *h, *y;
    int8_t* q;
    float *scale, *r;
    uint64_t rows, ldx, ldres, ldh, ldy, ldq;
    uint32_t cols;
    float eps;
};
struct NormGradArgs {
    const void *dy, *h, *dres;
    const float *w, *r;
    void* dx;
    float* part;                   // gridDim.x lines of `cols` sums, or nullptr
    uint64_t rows, lddy, ldh, lddres, lddx;
    uint32_t cols;
};

// Elements that a thread owns: G groups of eight neighbours (VEC: rows on 16-byte boundaries), group i from column
// 8 (thread + i threads); else single columns thread + j threads, so that a warp's accesses are contiguous wherever rows start.
template <bool VEC> __device__ __forceinline__ uint32_t column_of(uint32_t thread, uint32_t threads, uint32_t j) {
    return VEC ? (thread + (j >> 3) * threads) * 8 + (j & 7) : thread + j * threads;
}
template <typename T> __device__ __forceinline__ float load_one(const T* p) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(load4_bits(p));
    else return unpack2<T>(load2_bits(p)).x;
}
// Eight elements of a row: group i of the thread, zero beyond the row.
template <typename T, bool VEC>
__device__ __forceinline__ void load_group(const T* row, uint32_t thread, uint32_t threads, uint32_t i, uint32_t cols, float (&v)[8]) {
    if constexpr (VEC) {
        const uint32_t c = (thread + i * threads) * 8;
        widen8(c < cols ? fetch_raw8<T, true>(row, c, cols) : zero_raw8<T>(), v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t c = column_of<false>(thread, threads, 8 * i + j);
            v[j] = c < cols ? load_one<T>(row + c) : 0.f;
        }
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_group(T* row, uint32_t thread, uint32_t threads, uint32_t i, uint32_t cols, const float (&v)[8]) {
    const uint32_t c0 = column_of<VEC>(thread, threads, 8 * i);
    if (VEC && c0 + 8 <= cols) {
        store8(row + c0, v);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t c = column_of<VEC>(thread, threads, 8 * i + j);
        if (c < cols) row[c] = from_f32<T>(v[j]);
    }
}
// Rounded to T, as it is stored.
template <typename T> __device__ __forceinline__ float rounded(float v) { return to_f32(from_f32<T>(v)); }

// The sum and the largest bit pattern over the threads of a row; `half` alternates from row to row, so that one barrier a row does.
struct RowSums {
    float sum[2][32];
    uint32_t top[2][32];
};
template <bool TOP> __device__ __forceinline__ void row_meet(RowSums& sh, uint32_t half, float& sum, uint32_t& top) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(kFullMask, sum, d);
    if (TOP) top = __reduce_max_sync(kFullMask, top);
    if (blockDim.x > 32) {
        const uint32_t lane = threadIdx.x & 31, warps = blockDim.x >> 5;
        if (lane == 0) {
            sh.sum[half][threadIdx.x >> 5] = sum;
            if (TOP) sh.top[half][threadIdx.x >> 5] = top;
        }
        __syncthreads();
        sum = lane < warps ? sh.sum[half][lane] : 0.f;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(kFullMask, sum, d);
        if (TOP) top = __reduce_max_sync(kFullMask, lane < warps ? sh.top[half][lane] : 0u);
    }
}

// ---- forward -----------------------------------------------------------------------------------------
// blockDim.x threads share a row and hold all of it; blockDim.y rows at a time (more than one only where a row is one warp).
template <typename T, bool VEC, int G>
__global__ void __launch_bounds__(1024) norm_kernel(const __grid_constant__ NormArgs a) {
    __shared__ RowSums sh;
    const uint32_t me = threadIdx.x, n = blockDim.x;
    grid_wait();
    grid_go();
    float w[G][8];
#pragma unroll
    for (int i = 0; i < G; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t c = column_of<VEC>(me, n, 8 * i + j);
            w[i][j] = c < a.cols ? load_f32(a.w + c) : 0.f;
        }
    const float cols = (float)a.cols;
    const uint32_t padded = (a.cols + 15) / 16 * 16;
    uint32_t half = 0;
    for (uint64_t row = (uint64_t)blockIdx.x * blockDim.y + threadIdx.y; row < a.rows; row += (uint64_t)gridDim.x * blockDim.y, half ^= 1) {
        float h[G][8];
        float sum = 0.f;
        uint32_t top = 0;
        const T* x = static_cast<const T*>(a.x) + row * a.ldx;
#pragma unroll
        for (int i = 0; i < G; ++i) load_group<T, VEC>(x, me, n, i, a.cols, h[i]);
        if (a.residual) {
            const T* res = static_cast<const T*>(a.residual) + row * a.ldres;
            float v[G][8];
#pragma unroll
            for (int i = 0; i < G; ++i) load_group<T, VEC>(res, me, n, i, a.cols, v[i]);
#pragma unroll
            for (int i = 0; i < G; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] = rounded<T>(__fadd_rn(h[i][j], v[i][j]));
        }
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sum = __fmaf_rn(h[i][j], h[i][j], sum);
                top = max(top, __float_as_uint(__fmul_rn(h[i][j], w[i][j])) & 0x7FFFFFFFu);
            }
        row_meet<true>(sh, half, sum, top);
        const float r = __frsqrt_rn(__fadd_rn(__fdiv_rn(sum, cols), a.eps));
        if (me == 0 && a.r) a.r[row] = r;
        if (a.h) {
            T* out = static_cast<T*>(a.h) + row * a.ldh;
#pragma unroll
            for (int i = 0; i < G; ++i) store_group<T, VEC>(out, me, n, i, a.cols, h[i]);
        }
        if (a.y) {
            T* out = static_cast<T*>(a.y) + row * a.ldy;
#pragma unroll
            for (int i = 0; i < G; ++i) {
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = __fmul_rn(__fmul_rn(h[i][j], r), w[i][j]);
                store_group<T, VEC>(out, me, n, i, a.cols, y);
            }
        }
        if (a.q) {
            const LineScale s = line_scale(top);
            if (me == 0) a.scale[row] = __fmul_rn(s.scale, r);
            int8_t* out = a.q + row * a.ldq;
#pragma unroll
            for (int i = 0; i < G; ++i) {
                float t[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] = __fmul_rn(h[i][j], w[i][j]);
                const uint2 code = code8<false>(t, s.inv, DrawArgs{}, DrawRow{}, 0);
                if constexpr (VEC) {
                    const uint32_t c = column_of<VEC>(me, n, 8 * i);
                    if (c < padded) *reinterpret_cast<uint2*>(out + c) = code;
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t c = column_of<VEC>(me, n, 8 * i + j);
                        if (c < padded) out[c] = (int8_t)((j < 4 ? code.x : code.y) >> (8 * (j & 3)));
                    }
                }
            }
        }
    }
}

// Rows longer than a block holds: read twice, the second time from the caches.  Where h is written it is what the second pass
// reads (it may have replaced an input).
template <typename T>
__global__ void __launch_bounds__(1024) norm_long_kernel(const __grid_constant__ NormArgs a) {
    __shared__ RowSums sh;
    grid_wait();
    grid_go();
    const float cols = (float)a.cols;
    const uint32_t padded = (a.cols + 15) / 16 * 16;
    uint32_t half = 0;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, half ^= 1) {
        const T* x = static_cast<const T*>(a.x) + row * a.ldx;
        const T* res = a.residual ? static_cast<const T*>(a.residual) + row * a.ldres : nullptr;
        T* out_h = a.h ? static_cast<T*>(a.h) + row * a.ldh : nullptr;
        const auto element = [&](uint32_t c) {
            const float v = load_one<T>(x + c);
            return res ? rounded<T>(__fadd_rn(v, load_one<T>(res + c))) : v;
        };
        float sum = 0.f;
        uint32_t top = 0;
        for (uint32_t c = threadIdx.x; c < a.cols; c += 1024) {
            const float h = element(c);
            if (out_h) out_h[c] = from_f32<T>(h);
            sum = __fmaf_rn(h, h, sum);
            top = max(top, __float_as_uint(__fmul_rn(h, load_f32(a.w + c))) & 0x7FFFFFFFu);
        }
        row_meet<true>(sh, half, sum, top);
        const float r = __frsqrt_rn(__fadd_rn(__fdiv_rn(sum, cols), a.eps));
        const LineScale s = line_scale(top);
        if (threadIdx.x == 0) {
            if (a.r) a.r[row] = r;
            if (a.q) a.scale[row] = __fmul_rn(s.scale, r);
        }
        T* out_y = a.y ? static_cast<T*>(a.y) + row * a.ldy : nullptr;
        if (!out_y && !a.q) continue;
        for (uint32_t c = threadIdx.x; c < (a.q ? padded : a.cols); c += 1024) {
            const bool in = c < a.cols;
            const float h = !in ? 0.f : out_h ? to_f32(out_h[c]) : element(c), w = in ? load_f32(a.w + c) : 0.f;
            if (out_y && in) out_y[c] = from_f32<T>(__fmul_rn(__fmul_rn(h, r), w));
            if (a.q) a.q[row * a.ldq + c] = s.inv == 0.f ? 0 : (int8_t)code_bits<false>(__fmul_rn(h, w), s.inv, 0);
        }
    }
}

// ---- gradient ----------------------------------------------------------------------------------------
// With g = dy w: dx = r (g - h r^2 mean(g h)) + dres; dw = sum of dy h r over the rows.  A block adds up its rows' share of dw in
// registers and leaves it in `part`; a second kernel adds the blocks' shares, always in the same order.
template <typename T, bool VEC, int G>
__global__ void __launch_bounds__(G == 1 ? 512 : 1024) norm_grad_kernel(const __grid_constant__ NormGradArgs a) {
    __shared__ RowSums sh;
    __shared__ float sums[G == 1 ? 8 : 1][256];             // blocks of eight one-warp rows
    const uint32_t me = threadIdx.x, n = blockDim.x;
    grid_wait();
    grid_go();
    float w[G][8], dw[G][8] = {};
#pragma unroll
    for (int i = 0; i < G; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t c = column_of<VEC>(me, n, 8 * i + j);
            w[i][j] = c < a.cols ? load_f32(a.w + c) : 0.f;
        }
    const float cols = (float)a.cols;
    uint32_t half = 0, none = 0;
    for (uint64_t row = (uint64_t)blockIdx.x * blockDim.y + threadIdx.y; row < a.rows; row += (uint64_t)gridDim.x * blockDim.y, half ^= 1) {
        float dy[G][8], h[G][8];
        const T *pdy = static_cast<const T*>(a.dy) + row * a.lddy, *ph = static_cast<const T*>(a.h) + row * a.ldh;
        const float r = load_f32(a.r + row);
#pragma unroll
        for (int i = 0; i < G; ++i) {
            load_group<T, VEC>(pdy, me, n, i, a.cols, dy[i]);
            load_group<T, VEC>(ph, me, n, i, a.cols, h[i]);
        }
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dw[i][j] = __fmaf_rn(dy[i][j], __fmul_rn(h[i][j], r), dw[i][j]);
                dy[i][j] = __fmul_rn(dy[i][j], w[i][j]);
                dot = __fmaf_rn(dy[i][j], h[i][j], dot);
            }
        if (!a.dx) continue;
        row_meet<false>(sh, half, dot, none);
        const float along = __fdiv_rn(__fmul_rn(__fmul_rn(r, r), dot), cols);
        const T* pres = a.dres ? static_cast<const T*>(a.dres) + row * a.lddres : nullptr;
        T* out = static_cast<T*>(a.dx) + row * a.lddx;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            float v[8], res[8];
            if (pres) load_group<T, VEC>(pres, me, n, i, a.cols, res);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = __fmul_rn(r, __fmaf_rn(-h[i][j], along, dy[i][j]));
                if (pres) v[j] = __fadd_rn(v[j], res[j]);
            }
            store_group<T, VEC>(out, me, n, i, a.cols, v);
        }
    }
    if (!a.part) return;
    float* part = a.part + (uint64_t)blockIdx.x * a.cols;
    if constexpr (G == 1) {
        if (blockDim.y > 1) {
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[threadIdx.y][me + 32 * j] = dw[0][j];
            __syncthreads();
            const uint32_t c = column_of<VEC>(me, 32, threadIdx.y);
            if (c < a.cols) {
                float s = 0.f;
                for (uint32_t y = 0; y < blockDim.y; ++y) s += sums[y][me + 32 * threadIdx.y];
                part[c] = s;
            }
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < G; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t c = column_of<VEC>(me, n, 8 * i + j);
            if (c < a.cols) part[c] = dw[i][j];
        }
}

// Rows longer than a block holds, dx: read twice.
template <typename T>
__global__ void __launch_bounds__(1024) norm_grad_long_kernel(const __grid_constant__ NormGradArgs a) {
    __shared__ RowSums sh;
    grid_wait();
    grid_go();
    const float cols = (float)a.cols;
    uint32_t half = 0, none = 0;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, half ^= 1) {
        const T *pdy = static_cast<const T*>(a.dy) + row * a.lddy, *ph = static_cast<const T*>(a.h) + row * a.ldh;
        const T* pres = a.dres ? static_cast<const T*>(a.dres) + row * a.lddres : nullptr;
        const float r = load_f32(a.r + row);
        float dot = 0.f;
        for (uint32_t c = threadIdx.x; c < a.cols; c += 1024) dot = __fmaf_rn(__fmul_rn(load_one<T>(pdy + c), load_f32(a.w + c)), load_one<T>(ph + c), dot);
        row_meet<false>(sh, half, dot, none);
        const float along = __fdiv_rn(__fmul_rn(__fmul_rn(r, r), dot), cols);
        T* out = static_cast<T*>(a.dx) + row * a.lddx;
        for (uint32_t c = threadIdx.x; c < a.cols; c += 1024) {
            const float g = __fmul_rn(load_one<T>(pdy + c), load_f32(a.w + c));
            float v = __fmul_rn(r, __fmaf_rn(-load_one<T>(ph + c), along, g));
            if (pres) v = __fadd_rn(v, load_one<T>(pres + c));
            out[c] = from_f32<T>(v);
        }
    }
}
// dw of long rows: a thread a column, a block row (blockIdx.y) a share of the rows.
template <typename T>
__global__ void __launch_bounds__(256) norm_grad_long_dw_kernel(const __grid_constant__ NormGradArgs a) {
    grid_wait();
    grid_go();
    const uint64_t c = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    const uint64_t r0 = a.rows * blockIdx.y / gridDim.y, r1 = a.rows * (blockIdx.y + 1) / gridDim.y;
    const T *pdy = static_cast<const T*>(a.dy) + c, *ph = static_cast<const T*>(a.h) + c;
    float s = 0.f;
#pragma unroll 4
    for (uint64_t row = r0; row < r1; ++row) s = __fmaf_rn(load_one<T>(pdy + row * a.lddy), __fmul_rn(load_one<T>(ph + row * a.ldh), load_f32(a.r + row)), s);
    a.part[blockIdx.y * (uint64_t)a.cols + c] = s;
}

// dw from the shares: 32 columns a block, eight warps each a part of the shares.
__global__ void __launch_bounds__(256) norm_sum_kernel(const float* part, uint32_t shares, uint64_t cols, float* dw) {
    __shared__ float sh[8][32];
    grid_wait();
    grid_go();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint64_t c = (uint64_t)blockIdx.x * 32 + lane;
    const uint32_t k0 = shares * warp / 8, k1 = shares * (warp + 1) / 8;
    float s = 0.f;
    if (c < cols) {
#pragma unroll 8
        for (uint32_t k = k0; k < k1; ++k) s += load_f32(part + k * cols + c);
    }
    sh[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < cols) {
#pragma unroll
        for (int i = 1; i < 8; ++i) s += sh[i][lane];
        dw[c] = s;
    }
}

// ---- host ------------------------------------------------------------------------------------------
constexpr uint64_t kHeld = 16384;                          // columns that a block of 1024 threads holds, 16 each
// Threads of a row and rows of a block.
dim3 norm_block(uint64_t cols, int groups) {
    const uint64_t t = ((cols + 7) / 8 + groups - 1) / groups;
    return t <= 32 ? dim3(32, 8) : dim3((unsigned)((t + 31) / 32 * 32), 1);
}
// One group of eight a thread up to 4096 columns, two above.
int norm_groups(uint64_t cols) { return cols <= 4096 ? 1 : 2; }
// Blocks: rows, or as many as the SMs hold at once.
unsigned norm_grid(uint64_t rows, dim3 block, uint64_t threads_sm) {
    const uint64_t want = (rows + block.y - 1) / block.y, cap = (uint64_t)sm_count_now() * (threads_sm / (block.x * block.y) > 0 ? threads_sm / (block.x * block.y) : 1);
    return (unsigned)(want < cap ? want : cap);
}
// Blocks of the gradient, each with a share of dw: of a B200's SMs, not of the current device's, since the size of scratch follows from them.
uint64_t grad_shares(uint64_t rows, uint64_t cols) {
    if (cols > kHeld) {
        const uint64_t most = (rows + 63) / 64;            // 64 rows to a share at least
        return most < 64 ? most : 64;
    }
    const dim3 b = norm_block(cols, norm_groups(cols));
    const uint64_t want = (rows + b.y - 1) / b.y, per_sm = 1024 / (b.x * b.y) > 0 ? 1024 / (b.x * b.y) : 1, cap = 148 * (per_sm < 4 ? per_sm : 4);
    return want < cap ? want : cap;
}

bool row_vec(const void* p, size_t e, uint64_t rows, uint64_t ld) { return !p || (aligned(p, 16) && (rows == 1 || ld * e % 16 == 0)); }

template <typename T> cudaError_t launch_norm(const NormArgs& a, cudaStream_t st) {
    if (a.cols > kHeld) return launch_layer(norm_long_kernel<T>, norm_grid(a.rows, dim3(1024), 2048), 1024, 0, 1, st, a);
    const size_t e = sizeof(T);
    const bool vec = row_vec(a.x, e, a.rows, a.ldx) && row_vec(a.residual, e, a.rows, a.ldres) && row_vec(a.h, e, a.rows, a.ldh) && row_vec(a.y, e, a.rows, a.ldy);
    const int g = norm_groups(a.cols);
    const dim3 block = norm_block(a.cols, g);
    const auto kernel = g == 1 ? (vec ? norm_kernel<T, true, 1> : norm_kernel<T, false, 1>) : (vec ? norm_kernel<T, true, 2> : norm_kernel<T, false, 2>);
    return launch_layer(kernel, norm_grid(a.rows, block, 1024), block, 0, 1, st, a);
}

template <typename T> cudaError_t launch_norm_grad(const NormGradArgs& a, float* dw, cudaStream_t st) {
    const uint64_t shares = grad_shares(a.rows, a.cols);
    cudaError_t err = cudaSuccess;
    if (a.cols > kHeld) {
        if (a.dx) err = launch_layer(norm_grad_long_kernel<T>, norm_grid(a.rows, dim3(1024), 2048), 1024, 0, 1, st, a);
        if (err == cudaSuccess && dw) err = launch_layer(norm_grad_long_dw_kernel<T>, dim3((a.cols + 255) / 256, (unsigned)shares), 256, 0, 1, st, a);
    } else {
        const size_t e = sizeof(T);
        const bool vec = row_vec(a.dy, e, a.rows, a.lddy) && row_vec(a.h, e, a.rows, a.ldh) && row_vec(a.dres, e, a.rows, a.lddres) && row_vec(a.dx, e, a.rows, a.lddx);
        const int g = norm_groups(a.cols);
        const auto kernel = g == 1 ? (vec ? norm_grad_kernel<T, true, 1> : norm_grad_kernel<T, false, 1>)
                                   : (vec ? norm_grad_kernel<T, true, 2> : norm_grad_kernel<T, false, 2>);
        err = launch_layer(kernel, (unsigned)shares, norm_block(a.cols, g), 0, 1, st, a);
    }
    if (err != cudaSuccess || !dw) return err;
    return launch_layer(norm_sum_kernel, (unsigned)((a.cols + 31) / 32), 256, 0, 1, st, a.part, (uint32_t)shares, (uint64_t)a.cols, dw);
}

}  // namespace
}  // namespace tng

using namespace tng;

extern "C" {

tng_status tng_rmsnorm(const void* x_dev, tng_dtype type, uint64_t rows, uint64_t cols, uint64_t ldx, const void* residual_dev, uint64_t ldres,
                       const float* w_dev, float eps, void* h_dev, uint64_t ldh, void* y_dev, uint64_t ldy, int8_t* q_dev, uint64_t ldq,
                       float* scale_dev, float* r_dev, void* stream) {
    if (!type_ok(type) || cols < 1 || !dims_ok(rows, cols) || !(eps >= 0x1p-126f && eps <= 3.402823466e38f)) return TNG_ERR_INVALID_ARG;
    if (rows == 0) return TNG_OK;
    if (!matrix_ok(x_dev, type, cols, ldx) || !w_dev || !aligned(w_dev, 4) || !aligned(r_dev, 4) ||
        (residual_dev && !matrix_ok(residual_dev, type, cols, ldres)) || (h_dev && !matrix_ok(h_dev, type, cols, ldh)) ||
        (y_dev && !matrix_ok(y_dev, type, cols, ldy)) || (q_dev && (!codes_ok(q_dev, cols, ldq) || !scale_dev || !aligned(scale_dev, 4))))
        return TNG_ERR_INVALID_ARG;
    const NormArgs a{x_dev, residual_dev, w_dev, h_dev, y_dev, q_dev, scale_dev, r_dev, rows, ldx, ldres, ldh, ldy, ldq, (uint32_t)cols, eps};
    return layer_status(with_type(type, [&](auto t) { return launch_norm<decltype(t)>(a, static_cast<cudaStream_t>(stream)); }));
}

size_t tng_rmsnorm_grad_scratch_bytes(uint64_t rows, uint64_t cols) {
    if (rows == 0 || cols == 0) return 256;
    return (size_t)((grad_shares(rows, cols) * cols * 4 + 255) / 256 * 256);
}

tng_status tng_rmsnorm_grad(const void* dy_dev, uint64_t lddy, const void* h_dev, uint64_t ldh, tng_dtype type, uint64_t rows, uint64_t cols,
                            const float* w_dev, const float* r_dev, const void* dres_dev, uint64_t lddres, void* dx_dev, uint64_t lddx,
                            float* dw_dev, void* scratch_dev, void* stream) {
    if (!type_ok(type) || cols < 1 || !dims_ok(rows, cols) || !aligned(dw_dev, 4)) return TNG_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0) return layer_status(dw_dev ? cudaMemsetAsync(dw_dev, 0, cols * 4, st) : cudaSuccess);
    if (!dx_dev && !dw_dev) return TNG_OK;
    if (!matrix_ok(dy_dev, type, cols, lddy) || !matrix_ok(h_dev, type, cols, ldh) || !w_dev || !aligned(w_dev, 4) || !r_dev || !aligned(r_dev, 4) ||
        (dres_dev && !matrix_ok(dres_dev, type, cols, lddres)) || (dx_dev && !matrix_ok(dx_dev, type, cols, lddx)) ||
        (dw_dev && (!scratch_dev || !aligned(scratch_dev, 256))))
        return TNG_ERR_INVALID_ARG;
    const NormGradArgs a{dy_dev, h_dev, dres_dev, w_dev, r_dev, dx_dev, dw_dev ? static_cast<float*>(scratch_dev) : nullptr,
                         rows, lddy, ldh, lddres, lddx, (uint32_t)cols};
    return layer_status(with_type(type, [&](auto t) { return launch_norm_grad<decltype(t)>(a, dw_dev, st); }));
}

}  // extern "C"
