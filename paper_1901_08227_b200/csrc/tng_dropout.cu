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
    uint32_t lanes_log;    // log2 of the threads that share a segment of a row
    float inv_keep;
};

__device__ __forceinline__ float kept(float x, uint32_t word, const DropArgs& a) {
    return (word >= a.threshold && !a.none) ? __fmul_rn(x, a.inv_keep) : 0.f;
}

template <typename T> __device__ __forceinline__ Raw8<T> load_stream8(const T* p) {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.w[i] = load16_once(reinterpret_cast<const uint4*>(p) + i);
    return r;
}

// Eight elements: mask, scale, residual, store.
template <typename T, bool RES>
__device__ __forceinline__ void drop8(const Raw8<T>& rx, const Raw8<T>& rr, T* py, uint64_t column, const DrawRow& dr, const DropArgs& a) {
    const uint4 w0 = draw_words(a.draw, dr, column), w1 = draw_words(a.draw, dr, column + kPhiloxMul0);
    const uint32_t w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
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
}

// Rows that start on 16-byte boundaries.  `lanes` threads (a power of two up to 32) take a segment of 32 lanes columns of
// a row: four vectors of eight columns a thread, `lanes` vectors apart, their loads issued together.  WARP: 32 lanes (rows
// of 1024 columns and up), so that the distances are constants.  Bound by issue slots as much as by memory: a wide
// multiply takes three of them, 72 slots of Philox for four elements (after the two hoisted ones), so addresses, the row's
// part of Philox and the walk over (row, segment) are paid once in 32 elements.  16384 x 8192 bf16 with a residual 128 us
// (6.3 TB/s), 8192 x 8192 fp16 without 56 us (4.8 TB/s), both in short bursts; call after call 145 and 59 us at the
// power-limited clock.
template <typename T, bool RES, bool WARP>
__global__ void __launch_bounds__(kThreads, 3) dropout_kernel(const T* x, const T* res, T* y, const __grid_constant__ DropArgs a) {
    constexpr int kVec = 4;
    grid_wait();
    grid_go();
    const uint32_t lanes_log = WARP ? 5u : a.lanes_log, cols = (uint32_t)a.cols;
    const uint32_t lane = threadIdx.x & ((1u << lanes_log) - 1u), span = 8u << lanes_log;          // columns from one vector to the next
    const uint32_t segs = (cols - 1) / (kVec * span) + 1;
    const uint64_t units = a.rows * segs, stride = ((uint64_t)gridDim.x * kThreads) >> lanes_log;
    uint64_t unit = ((uint64_t)blockIdx.x * kThreads + threadIdx.x) >> lanes_log;
    uint32_t row = (uint32_t)(unit / segs), seg = (uint32_t)(unit - (uint64_t)row * segs);
    const uint32_t drow = (uint32_t)(stride / segs), dseg = (uint32_t)(stride - (uint64_t)drow * segs);
    const uint64_t next = draw_column(span >> 2);
    for (; unit < units; unit += stride) {
        const uint32_t c = seg * (kVec * span) + lane * 8;
        const T* px = x + row * a.ldx + c;
        const T* pr = RES ? res + row * a.ldr + c : nullptr;
        T* py = y + row * a.ldy + c;
        const DrawRow dr = draw_row(a.draw, row);
        uint64_t column = draw_column(c >> 2);
        Raw8<T> rx[kVec], rr[kVec];
        if (c + (kVec - 1) * span + 8 <= cols) {
#pragma unroll
            for (int u = 0; u < kVec; ++u) {
                rx[u] = load_stream8(px + u * span);
                if (RES) rr[u] = load_stream8(pr + u * span);
            }
#pragma unroll
            for (int u = 0; u < kVec; ++u, column += next) drop8<T, RES>(rx[u], rr[u], py + u * span, column, dr, a);
        } else {                                           // the row ends in this segment
#pragma unroll 1
            for (uint32_t u = 0; u < kVec && c + u * span < cols; ++u, column += next) {
                const uint32_t left = cols - (c + u * span);
                if (left >= 8) {
                    rx[0] = load_stream8(px + u * span);
                    if (RES) rr[0] = load_stream8(pr + u * span);
                    drop8<T, RES>(rx[0], rr[0], py + u * span, column, dr, a);
                } else {
                    for (uint32_t j = 0; j < left; ++j) {
                        const uint4 w = draw_words(a.draw, dr, column + (j < 4 ? 0u : kPhiloxMul0));
                        const uint32_t word = j & 2 ? (j & 1 ? w.w : w.z) : (j & 1 ? w.y : w.x);
                        const float v = kept(to_f32(px[u * span + j]), word, a);
                        py[u * span + j] = from_f32<T>(RES ? __fadd_rn(to_f32(pr[u * span + j]), v) : v);
                    }
                }
            }
        }
        row += drow;
        seg += dseg;
        if (seg >= segs) { seg -= segs; ++row; }
    }
}

// Any alignment: a warp takes VEC times 128 columns of a row, one Philox call a lane and 128, and turns the four keep
// bits a lane drew into four ballots; loads and stores then run over the columns lane by lane, so that they are
// contiguous across the warp wherever the row starts.  (Eight scalar accesses by one thread would touch every sector of
// the warp's span once an access.)  VEC = 1 has the shortest path for a thread: the one for small arrays.
// 4097 x 2501 fp32: 20 us, 4.1 TB/s (16 us with the arrays in the L2 cache).
template <typename T, bool RES, bool WHOLE>
__device__ __forceinline__ void drop128(T* py, uint32_t left, uint32_t lane, uint64_t column, const DrawRow& dr, const float (&v)[4], const float (&r)[4], const DropArgs& a) {
    const uint4 w = draw_words(a.draw, dr, column);
    const uint32_t b0 = __ballot_sync(kFullMask, w.x >= a.threshold), b1 = __ballot_sync(kFullMask, w.y >= a.threshold);
    const uint32_t b2 = __ballot_sync(kFullMask, w.z >= a.threshold), b3 = __ballot_sync(kFullMask, w.w >= a.threshold);
    // column 32 q + lane of the 128 is word lane % 4 of lane 8 q + lane / 4
    const uint32_t lo = lane & 1 ? b1 : b0, hi = lane & 1 ? b3 : b2;
    const uint32_t bits = a.none ? 0u : (lane & 2 ? hi : lo) >> (lane >> 2);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float k = bits >> (8 * q) & 1u ? __fmul_rn(v[q], a.inv_keep) : 0.f;
        if (WHOLE || 32u * q + lane < left) py[32 * q] = from_f32<T>(RES ? __fadd_rn(r[q], k) : k);
    }
}
template <typename T, bool RES, int VEC>
__global__ void __launch_bounds__(kThreads, VEC == 1 ? 4 : 3) dropout_any_kernel(const T* x, const T* res, T* y, const __grid_constant__ DropArgs a) {
    grid_wait();
    grid_go();
    const uint32_t lane = threadIdx.x & 31, cols = (uint32_t)a.cols, segs = (cols - 1) / (128 * VEC) + 1;
    const uint64_t units = a.rows * segs, stride = (uint64_t)gridDim.x * (kThreads / 32);
    uint64_t unit = (uint64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    uint32_t row = (uint32_t)(unit / segs), seg = (uint32_t)(unit - (uint64_t)row * segs);
    const uint32_t drow = (uint32_t)(stride / segs), dseg = (uint32_t)(stride - (uint64_t)drow * segs);
    const uint64_t next = draw_column(32);
    for (; unit < units; unit += stride) {
        const uint32_t c = seg * (128 * VEC);              // first column of the warp's segment
        const T* px = x + row * a.ldx + c + lane;
        const T* pr = RES ? res + row * a.ldr + c + lane : nullptr;
        T* py = y + row * a.ldy + c + lane;
        const DrawRow dr = draw_row(a.draw, row);
        uint64_t column = draw_column(c / 4 + lane);
        if (cols - c >= 128 * VEC) {
            float v[VEC][4], r[VEC][4];
#pragma unroll
            for (int u = 0; u < VEC; ++u)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    v[u][q] = to_f32(px[128 * u + 32 * q]);
                    r[u][q] = RES ? to_f32(pr[128 * u + 32 * q]) : 0.f;
                }
#pragma unroll
            for (int u = 0; u < VEC; ++u, column += next)
                drop128<T, RES, true>(py + 128 * u, 128, lane, column, dr, v[u], r[u], a);
        } else {
#pragma unroll 1
            for (uint32_t at = 0; at < cols - c; at += 128, column += next) {
                const uint32_t left = cols - c - at;
                float v[4], r[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const bool in = 32u * q + lane < left;
                    v[q] = in ? to_f32(px[at + 32 * q]) : 0.f;
                    r[q] = RES && in ? to_f32(pr[at + 32 * q]) : 0.f;
                }
                drop128<T, RES, false>(py + at, left, lane, column, dr, v, r, a);
            }
        }
        row += drow;
        seg += dseg;
        if (seg >= segs) { seg -= segs; ++row; }
    }
}

template <typename T>
cudaError_t launch_dropout(const void* x, const void* res, void* y, const DropArgs& a, cudaStream_t st) {
    const T *px = static_cast<const T*>(x), *pr = static_cast<const T*>(res);
    T* py = static_cast<T*>(y);
    const uint64_t e = sizeof(T);
    const bool vec = aligned(x, 16) && aligned(y, 16) && (!res || aligned(res, 16)) &&
                     (a.rows == 1 || ((a.ldx * e) % 16 == 0 && (a.ldy * e) % 16 == 0 && (!res || (a.ldr * e) % 16 == 0)));
    // Small arrays (a wave of 128 columns a warp holds them) take the kernel with the least work a thread, whatever their
    // alignment: 16 x 1024 bf16 1.6 us, 2.4 us with 32 elements a thread.
    const uint64_t sms = (uint64_t)sm_count_now();
    const bool small = a.rows * ((a.cols + 127) / 128) <= sms * 32, warp = a.lanes_log == 5;
    const uint64_t span = 32ull << a.lanes_log;
    const uint64_t work = small ? a.rows * ((a.cols + 127) / 128) * 32
                          : vec ? a.rows * ((a.cols + span - 1) / span) << a.lanes_log : a.rows * ((a.cols + 511) / 512) * 32;
    const uint64_t want = (work + kThreads - 1) / kThreads, cap = sms * 8u;
    const unsigned grid = (unsigned)(want < cap ? want : cap);
    const auto kernel = small ? (res ? dropout_any_kernel<T, true, 1> : dropout_any_kernel<T, false, 1>)
                        : !vec ? (res ? dropout_any_kernel<T, true, 4> : dropout_any_kernel<T, false, 4>)
                        : warp ? (res ? dropout_kernel<T, true, true> : dropout_kernel<T, false, true>)
                               : (res ? dropout_kernel<T, true, false> : dropout_kernel<T, false, false>);
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
    a.lanes_log = 0;
    while (a.lanes_log < 5 && (32ull << a.lanes_log) < cols) ++a.lanes_log;
    a.none = grid24 >= (1u << 24);
    a.threshold = a.none ? 0u : (uint32_t)grid24 << 8;
    a.inv_keep = a.none ? 0.f : 1.0f / (1.0f - p);
    const cudaError_t e = with_type(type, [&](auto t) {
        return launch_dropout<decltype(t)>(x_dev, residual_dev, y_dev, a, static_cast<cudaStream_t>(stream));
    });
    return layer_status(e);
}
