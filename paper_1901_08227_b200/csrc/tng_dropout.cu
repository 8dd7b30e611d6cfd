// Dropout with the residual sum, y = residual + keep(x) / (1 - p), and its gradient (the same map of dy).
//
// The mask is a function of (seed, step, layer, row, column): every element's 24-bit uniform comes from
// Philox and is compared with p again in the backward pass, so nothing is stored between the two.
// u >= p on the 2^-24 grid is word >= ceil(p 2^24) 2^8 as integers: one compare an element.
//
// One read of each input, one write; bound by memory traffic, with the ten Philox rounds (20 wide
// multiplies and 20 three-input logic operations for four elements) next.
#include <math.h>

#include "tng_layers.cuh"

namespace tng {
namespace {

constexpr int kThreads = 256;

struct DropArgs {
    DrawArgs draw;
    uint64_t rows, cols, ldx, ldr, ldy;
    uint32_t threshold;    // keep when word >= threshold ...
    uint32_t none;         // ... unless everything is dropped (p = 1)
    float inv_keep;
};

__device__ __forceinline__ float kept(float x, uint32_t word, const DropArgs& a) {
    return (word >= a.threshold && !a.none) ? __fmul_rn(x, a.inv_keep) : 0.f;
}

template <typename T> __device__ __forceinline__ Raw8<T> load_stream8(const T* p) {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.w[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
    return r;
}

// Rows that start on 16-byte boundaries: a thread takes eight columns of a row at a time (two Philox
// calls), the groups of eight of all rows in one grid-stride sequence.  (row, group) advances by a fixed
// step, so no division in the loop.
template <typename T, bool RES>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const T* x, const T* res, T* y, const __grid_constant__ DropArgs a) {
    grid_wait();
    grid_go();
    const uint32_t per_row = (uint32_t)((a.cols + 7) / 8);
    const uint64_t total = a.rows * per_row, stride = (uint64_t)gridDim.x * kThreads;
    const uint64_t first = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    uint64_t row = first / per_row;
    uint32_t g = (uint32_t)(first - row * per_row);
    const uint64_t drow = stride / per_row;
    const uint32_t dg = (uint32_t)(stride - drow * per_row);
    for (uint64_t i = first; i < total; i += stride) {
        const uint64_t c = (uint64_t)g * 8;
        const T* px = x + row * a.ldx + c;
        const T* pr = RES ? res + row * a.ldr + c : nullptr;
        T* py = y + row * a.ldy + c;
        const bool whole = c + 8 <= a.cols;
        Raw8<T> rx, rr;
        if (whole) {
            rx = load_stream8(px);
            if (RES) rr = load_stream8(pr);
        }
        const uint4 w0 = draw_words(a.draw, 2 * g, (uint32_t)row), w1 = draw_words(a.draw, 2 * g + 1, (uint32_t)row);
        const uint32_t w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
        if (whole) {
            float v[8];
            widen8(rx, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = kept(v[j], w[j], a);
            if (RES) {
                float r[8];
                widen8(rr, r);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = __fadd_rn(r[j], v[j]);
            }
            store8(py, v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (c + j >= a.cols) break;
                const float v = kept(to_f32(px[j]), w[j], a);
                py[j] = from_f32<T>(RES ? __fadd_rn(to_f32(pr[j]), v) : v);
            }
        }
        row += drow;
        g += dg;
        if (g >= per_row) { g -= per_row; ++row; }
    }
}

// Any other alignment: a warp takes 128 columns of a row, one Philox call a lane, and turns the four keep
// bits a lane drew into four ballots; loads and stores then run over the columns lane by lane, so that
// they are contiguous across the warp wherever the row starts.  (Eight scalar accesses by one thread
// would touch every sector of the warp's span once an access.)
template <typename T, bool RES>
__global__ void __launch_bounds__(kThreads) dropout_any_kernel(const T* x, const T* res, T* y, const __grid_constant__ DropArgs a) {
    grid_wait();
    grid_go();
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t per_row = (uint32_t)((a.cols + 127) / 128);
    const uint64_t total = a.rows * per_row, stride = (uint64_t)gridDim.x * (kThreads / 32);
    const uint64_t first = (uint64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    uint64_t row = first / per_row;
    uint32_t g = (uint32_t)(first - row * per_row);
    const uint64_t drow = stride / per_row;
    const uint32_t dg = (uint32_t)(stride - drow * per_row);
    for (uint64_t i = first; i < total; i += stride) {
        const uint64_t c = (uint64_t)g * 128 + lane;
        const T* px = x + row * a.ldx;
        const T* pr = RES ? res + row * a.ldr : nullptr;
        float v[4], r[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const bool in = c + 32 * q < a.cols;
            v[q] = in ? to_f32(px[c + 32 * q]) : 0.f;
            r[q] = RES && in ? to_f32(pr[c + 32 * q]) : 0.f;
        }
        const uint4 w = draw_words(a.draw, 32 * g + lane, (uint32_t)row);
        const uint32_t b0 = __ballot_sync(kFullMask, w.x >= a.threshold), b1 = __ballot_sync(kFullMask, w.y >= a.threshold);
        const uint32_t b2 = __ballot_sync(kFullMask, w.z >= a.threshold), b3 = __ballot_sync(kFullMask, w.w >= a.threshold);
        // column 32 q + lane of the 128 is word lane % 4 of lane 8 q + lane / 4
        const uint32_t lo = lane & 1 ? b1 : b0, hi = lane & 1 ? b3 : b2;
        const uint32_t bits = (lane & 2 ? hi : lo) >> (lane >> 2);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (c + 32 * q >= a.cols) break;
            const float k = ((bits >> (8 * q)) & 1u) && !a.none ? __fmul_rn(v[q], a.inv_keep) : 0.f;
            y[row * a.ldy + c + 32 * q] = from_f32<T>(RES ? __fadd_rn(r[q], k) : k);
        }
        row += drow;
        g += dg;
        if (g >= per_row) { g -= per_row; ++row; }
    }
}

template <typename T>
cudaError_t launch_dropout(const void* x, const void* res, void* y, const DropArgs& a, cudaStream_t st) {
    const T *px = static_cast<const T*>(x), *pr = static_cast<const T*>(res);
    T* py = static_cast<T*>(y);
    const uint64_t e = sizeof(T);
    const bool vec = aligned(x, 16) && aligned(y, 16) && (!res || aligned(res, 16)) &&
                     (a.rows == 1 || ((a.ldx * e) % 16 == 0 && (a.ldy * e) % 16 == 0 && (!res || (a.ldr * e) % 16 == 0)));
    const uint64_t work = vec ? a.rows * ((a.cols + 7) / 8) : a.rows * ((a.cols + 127) / 128) * 32;
    const uint64_t want = (work + kThreads - 1) / kThreads, cap = (uint64_t)sm_count_now() * 8u;
    const unsigned grid = (unsigned)(want < cap ? want : cap);
    const auto kernel = vec ? (res ? dropout_kernel<T, true> : dropout_kernel<T, false>) : (res ? dropout_any_kernel<T, true> : dropout_any_kernel<T, false>);
    return launch_layer(kernel, grid, kThreads, 0, 1, st, px, pr, py, a);
}

}  // namespace
}  // namespace tng

using namespace tng;

extern "C" tng_status tng_dropout(const void* x_dev, tng_dtype type, uint64_t rows, uint64_t cols, uint64_t ldx,
                                  const void* residual_dev, uint64_t ldr, float p, const tng_draw* draw, void* y_dev,
                                  uint64_t ldy, void* stream) {
    if (!type_ok(type) || !draw || cols < 1 || !dims_ok(rows, cols) || !(p >= 0.f && p <= 1.f)) return TNG_ERR_INVALID_ARG;
    if (!draw_ok(draw, rows)) return TNG_ERR_INVALID_ARG;
    if (rows == 0) return TNG_OK;
    if (!matrix_ok(x_dev, type, cols, ldx) || !matrix_ok(y_dev, type, cols, ldy) ||
        (residual_dev && !matrix_ok(residual_dev, type, cols, ldr)))
        return TNG_ERR_INVALID_ARG;
    DropArgs a;
    a.draw = make_draw(*draw, kTagDropout);
    a.rows = rows; a.cols = cols; a.ldx = ldx; a.ldr = ldr; a.ldy = ldy;
    const uint64_t grid24 = (uint64_t)ceil((double)p * 16777216.0);    // exact: p has 24 significant bits
    a.none = grid24 >= (1u << 24);
    a.threshold = a.none ? 0u : (uint32_t)grid24 << 8;
    a.inv_keep = a.none ? 0.f : 1.0f / (1.0f - p);
    const cudaError_t e = with_type(type, [&](auto t) {
        return launch_dropout<decltype(t)>(x_dev, residual_dev, y_dev, a, static_cast<cudaStream_t>(stream));
    });
    return e == cudaSuccess ? TNG_OK : TNG_ERR_CUDA;
}
