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
// Both directions are bound by memory, as long as the instructions a thread spends on a row, whatever its elements (sums over the
// team, the root, quotients: about 80), are shared by enough of them: a thread has up to 32 elements of a row (16384 x 4096 bf16
// with 8: 92 us for y alone, bound by issue slots).  The threads of a row (a team) meet once a row.  Three ways to read rows:
//   kStaged   rows that start and end on 16-byte boundaries, of more than 1024 columns: a team of whole warps with a barrier of its own; the
//             rows are on their way into shared memory, by bulk copies, while others are worked on
//   kDirect   shorter ones: a team of 8, 16 or 32 lanes, which needs no barrier; an SM holds enough of them to keep memory busy (65536 x
//             64 bf16 with a copy a row: 29 us)
//   kApart    rows that start anywhere: single elements, neighbours by neighbouring lanes
// The weights stay in shared memory.  The border at 1024 columns, 2^25 elements, kDirect / kStaged in us, bf16 and fp32 (codes with a residual; y;
// gradient with dres):
//   512     45 / 45, 74 / 72       29 / 31, 51 / 52       63 / 69, 93 / 97
//   768     49 / 64, 72 / 74       29 / 45, 51 / 55       81 / 65, 99 / 114
//   1024    41 / 47, 74 / 76       25 / 33, 49 / 55       69 / 56, 89 / 93
//   1280    102 / 57, 115 / 74     78 / 39, 92 / 57       95 / 69, 112 / 99
//   2048    64 / 47, 78 / 74       45 / 33, 64 / 55       71 / 54, 93 / 91
// (16-bit gradients of 768 to 1024 columns would gain by the other side; one border serves all.)
#include <math_constants.h>

#include <type_traits>

#include "tng_codes.cuh"
#include "tng_pipeline.cuh"

namespace tng {
namespace {

struct NormArgs {
    const void *x, *residual;
    const float* w;
    void *h, *y;
    int8_t* q;
    float *scale, *r;
    uint64_t rows, ldx, ldres, ldh, ldy, ldq;
    uint32_t cols, stages;         // stages: rows of a team under way
    float eps, inv_cols;
};
struct NormGradArgs {
    const void *dy, *h, *dres;
    const float *w, *r;
    void* dx;
    float* part;                   // gridDim.x lines of `cols` sums, or nullptr
    uint64_t rows, lddy, ldh, lddres, lddx;
    uint32_t cols, stages, arrays; // arrays: staged ones, 2 (dy, h) or 3 (dres too)
    float inv_cols;
};

enum Mode { kApart = 0, kDirect = 1, kStaged = 2 };
// Elements that a thread owns: G groups of eight neighbours (VEC: all but kApart), group i from column 8 (thread + i threads); else
// single columns thread + j threads, so that a warp's accesses are contiguous wherever rows start.
template <bool VEC> __device__ __forceinline__ uint32_t column_of(uint32_t thread, uint32_t threads, uint32_t j) {
    return VEC ? (thread + (j >> 3) * threads) * 8 + (j & 7) : thread + j * threads;
}
// Arithmetic goes two values at a time, one instruction for both.  (Not the product and the sum that make a code: the compiler may turn
// such a pair into a fused operation, which rounds once and changed one code in two million.)
struct Eight {
    float2 v[4];
    __device__ __forceinline__ float at(int j) const { return j & 1 ? v[j >> 1].y : v[j >> 1].x; }
};
__device__ __forceinline__ float2 twice(float v) { return make_float2(v, v); }
template <typename T> __device__ __forceinline__ Eight widen(const Raw8<T>& r) {
    Eight e;
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) e.v[i] = make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
        else e.v[i] = unpack2<T>(w[i]);
    }
    return e;
}
template <typename T> __device__ __forceinline__ Raw8<T> narrow(const Eight& e) {
    Raw8<T> r;
    uint32_t* w = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            w[2 * i] = __float_as_uint(e.v[i].x);
            w[2 * i + 1] = __float_as_uint(e.v[i].y);
        } else {
            w[i] = pack2<T>(e.v[i].x, e.v[i].y);
        }
    }
    return r;
}
__device__ __forceinline__ Eight times(const Eight& a, const Eight& b) {
    Eight e;
#pragma unroll
    for (int i = 0; i < 4; ++i) e.v[i] = __fmul2_rn(a.v[i], b.v[i]);
    return e;
}
__device__ __forceinline__ Eight times(const Eight& a, float b) {
    Eight e;
#pragma unroll
    for (int i = 0; i < 4; ++i) e.v[i] = __fmul2_rn(a.v[i], twice(b));
    return e;
}
__device__ __forceinline__ Eight plus(const Eight& a, const Eight& b) {
    Eight e;
#pragma unroll
    for (int i = 0; i < 4; ++i) e.v[i] = __fadd2_rn(a.v[i], b.v[i]);
    return e;
}

template <typename T> __device__ __forceinline__ float load_one(const T* p) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(load4_bits(p));
    else return unpack2<T>(load2_bits(p)).x;
}
// Eight elements of a row as they lie in memory, columns thread + (8 i + j) threads; zero beyond the row.
template <typename T> __device__ __forceinline__ Raw8<T> load_apart(const T* row, uint32_t thread, uint32_t threads, uint32_t i, uint32_t cols) {
    const uint32_t c0 = column_of<false>(thread, threads, 8 * i);
    Raw8<T> r;
    uint32_t* w = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
    for (int j = 0; j < 8; j += 4 / (int)sizeof(T)) {
        const uint32_t c = c0 + j * threads;
        if constexpr (sizeof(T) == 4) w[j] = c < cols ? load4_bits(row + c) : 0u;
        else w[j / 2] = (c < cols ? load2_bits(row + c) : 0u) | (c + threads < cols ? load2_bits(row + c + threads) : 0u) << 16;
    }
    return r;
}
// Eight neighbours of a row in shared memory, which is filled up with zeros.
template <typename T> __device__ __forceinline__ Raw8<T> load_staged(uint32_t row, uint32_t thread, uint32_t threads, uint32_t i) {
    Raw8<T> r;
#pragma unroll
    for (int k = 0; k < (int)(sizeof(T) / 2); ++k) {
        const float4 v = lds128(row + (thread + i * threads) * 8 * (uint32_t)sizeof(T) + 16 * k);
        r.w[k] = make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w));
    }
    return r;
}
// Eight neighbours of a row in global memory that would fit the stages (a group of fp32 may be half inside).
template <typename T> __device__ __forceinline__ Raw8<T> load_together(const T* row, uint32_t thread, uint32_t threads, uint32_t i, uint32_t cols) {
    const uint32_t c0 = column_of<true>(thread, threads, 8 * i);
    Raw8<T> r = zero_raw8<T>();
#pragma unroll
    for (int k = 0; k < (int)(sizeof(T) / 2); ++k)
        if (c0 + 4 * k < cols) r.w[k] = load16(row + c0 + 4 * k);
    return r;
}
template <typename T, bool VEC> __device__ __forceinline__ Raw8<T> load_direct(const T* row, uint32_t thread, uint32_t threads, uint32_t i, uint32_t cols) {
    if constexpr (VEC) return load_together<T>(row, thread, threads, i, cols);
    else return load_apart<T>(row, thread, threads, i, cols);
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_group(T* row, uint32_t thread, uint32_t threads, uint32_t i, uint32_t cols, const Raw8<T>& r) {
    const uint32_t c0 = column_of<VEC>(thread, threads, 8 * i);
    if constexpr (VEC) {
#pragma unroll
        for (int k = 0; k < (int)(sizeof(T) / 2); ++k)
            if (c0 + 4 * k < cols) reinterpret_cast<uint4*>(row + c0)[k] = r.w[k];
    } else {
        const T* v = reinterpret_cast<const T*>(&r);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c0 + j * threads < cols) row[c0 + j * threads] = v[j];
    }
}
// x + residual rounded to the type.
template <typename T> __device__ __forceinline__ Raw8<T> rounded_sum(const Raw8<T>& x, const Raw8<T>& res) { return narrow<T>(plus(widen(x), widen(res))); }
template <typename T> __device__ __forceinline__ float rounded(float v) { return to_f32(from_f32<T>(v)); }
// Codes to nearest of eight values.
__device__ __forceinline__ uint2 codes_of(const Eight& t, float inv) {
    const float v[8] = {t.v[0].x, t.v[0].y, t.v[1].x, t.v[1].y, t.v[2].x, t.v[2].y, t.v[3].x, t.v[3].y};
    return code8<false>(v, inv, DrawArgs{}, DrawRow{}, 0);
}
template <typename T> __device__ __forceinline__ Raw8<T> all_nan() {
    Raw8<T> r;
#pragma unroll
    for (int k = 0; k < (int)(sizeof(T) / 2); ++k) r.w[k] = make_uint4(~0u, ~0u, ~0u, ~0u);
    return r;
}

// Rows on their way to a team: `stages` of them, each ARRAYS rows of
// memory at most (a null one is not copied) behind one another.  A wait that gives up makes the team's further rows NaN.
constexpr uint32_t kMostStages = 4, kMostTeams = 16;
template <typename T, int ARRAYS> struct RowStages {
    uint32_t data, bars, bytes, pitch, arrays, slot, parity;
    bool ok;
    // pitch: bytes of a row as the team reads it, zeros behind the row
    __device__ __forceinline__ RowStages(unsigned char* smem, uint64_t* bar, uint32_t cols, uint32_t pitch_, uint32_t stages, uint32_t arrays_)
        : bytes(cols * (uint32_t)sizeof(T)), pitch(pitch_), arrays(arrays_), slot(0), parity(0), ok(true) {
        unsigned char* mine = smem + threadIdx.y * stages * arrays * pitch;
        data = smem_u32(mine);
        bars = smem_u32(bar + threadIdx.y * kMostStages);
        for (uint32_t r = 0; r < stages * arrays; ++r)
            for (uint32_t at = bytes + 16 * threadIdx.x; at < pitch; at += 16 * blockDim.x) *reinterpret_cast<uint4*>(mine + r * pitch + at) = make_uint4(0u, 0u, 0u, 0u);
        if (threadIdx.x == 0) {
            for (uint32_t i = 0; i < stages; ++i) mbar_init(bars + 8 * i, 1);
            mbar_init_fence();
        }
        __syncthreads();
    }
    // (one thread)
    __device__ __forceinline__ void send(uint32_t stage, const T* const (&rows)[ARRAYS]) const {
        mbar_expect_tx(bars + 8 * stage, arrays * bytes);
        uint32_t at = data + stage * arrays * pitch;
#pragma unroll
        for (int i = 0; i < ARRAYS; ++i)
            if (rows[i]) {
                bulk_load(at, rows[i], bytes, bars + 8 * stage);
                at += pitch;
            }
    }
    // Address of the next row's first array.
    __device__ __forceinline__ uint32_t take() {
        if (ok && !mbar_wait(bars + 8 * slot, parity)) ok = false;
        return data + slot * arrays * pitch;
    }
    __device__ __forceinline__ void next(uint32_t stages) {
        if (++slot == stages) {
            slot = 0;
            parity ^= 1u;
        }
    }
    // After a failure nobody leaves before the copies have landed, or a wait has run out once more.
    __device__ __forceinline__ void leave(uint32_t stages) {
        if (!ok)
            for (uint32_t i = 0; i < stages; ++i) (void)mbar_wait_limited(bars + 8 * i, parity, kSpinLimit / kMostStages);
    }
};

// The sum and the largest bit pattern over a team; `half` alternates from row to row, so that one barrier a row does.
struct RowSums {
    float sum[2][32];
    uint32_t top[2][32];
};
__device__ __forceinline__ void team_meet() {
    if (blockDim.x > 32) asm volatile("bar.sync %0, %1;" ::"r"(threadIdx.y + 1), "r"(blockDim.x) : "memory");   // (at most 8 teams of more than a warp)
    else __syncwarp();
}
template <bool TOP> __device__ __forceinline__ void row_meet(RowSums& sh, uint32_t half, float& sum, uint32_t& top) {
    if (blockDim.x < 32) {                                 // several teams in a warp
        for (uint32_t d = blockDim.x >> 1; d > 0; d >>= 1) {
            sum += __shfl_xor_sync(kFullMask, sum, d);
            if (TOP) top = max(top, __shfl_xor_sync(kFullMask, top, d));
        }
        return;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(kFullMask, sum, d);
    if (TOP) top = __reduce_max_sync(kFullMask, top);
    if (blockDim.x > 32) {
        const uint32_t lane = threadIdx.x & 31, warps = blockDim.x >> 5, first = threadIdx.y * warps;
        if (lane == 0) {
            sh.sum[half][first + (threadIdx.x >> 5)] = sum;
            if (TOP) sh.top[half][first + (threadIdx.x >> 5)] = top;
        }
        team_meet();
        sum = lane < warps ? sh.sum[half][first + lane] : 0.f;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(kFullMask, sum, d);
        if (TOP) top = __reduce_max_sync(kFullMask, lane < warps ? sh.top[half][first + lane] : 0u);
    } else {
        team_meet();
    }
}
// The first row of a thread's warp, relative to its own: all lanes take part in every round, since teams of a warp meet together.
__device__ __forceinline__ uint32_t rows_ahead() { return blockDim.x < 32 ? threadIdx.y & (32 / blockDim.x - 1) : 0u; }
// Larger magnitude, NaN on top.
__device__ __forceinline__ float larger(float top, float v) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(fabsf(v)));
    return top;
}
// The weights in shared memory, zeros behind them up to what the team reads.  VEC: the first four of every eight columns, then the last
// four, so that lanes read 16 bytes each without bank conflicts; else as they are.
template <bool VEC> struct Weights {
    float* at;
    uint32_t groups;               // of eight
    __device__ __forceinline__ Weights(float* smem, uint32_t groups_) : at(smem), groups(groups_) {}
    __device__ __forceinline__ void fill(const float* w, uint32_t cols) const {
        for (uint32_t c = threadIdx.y * blockDim.x + threadIdx.x; c < groups * 8; c += blockDim.x * blockDim.y)
            at[VEC ? (c >> 2 & 1) * groups * 4 + (c >> 3) * 4 + (c & 3) : c] = c < cols ? load_f32(w + c) : 0.f;
    }
    // of group i of a thread
    __device__ __forceinline__ Eight get(uint32_t thread, uint32_t threads, uint32_t i) const {
        Eight e;
        if constexpr (VEC) {
            const uint32_t g = thread + i * threads;
            const float4 a = *reinterpret_cast<const float4*>(at + g * 4), b = *reinterpret_cast<const float4*>(at + (groups + g) * 4);
            e.v[0] = make_float2(a.x, a.y);
            e.v[1] = make_float2(a.z, a.w);
            e.v[2] = make_float2(b.x, b.y);
            e.v[3] = make_float2(b.z, b.w);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) e.v[j] = make_float2(at[thread + (8 * i + 2 * j) * threads], at[thread + (8 * i + 2 * j + 1) * threads]);
        }
        return e;
    }
};

// ---- forward -----------------------------------------------------------------------------------------
// blockDim.y teams of blockDim.x threads, G groups of eight elements a thread.  16384 x 8192 bf16 with a residual into codes: 154 us by itself, 161 to
// 170 in long runs (0.89 to 0.84 of the copy rate); y alone 100 us (0.82); 65536 x 128 into codes: 20 us; rows that start anywhere, 16384 x 1001 with
// a residual into codes: fp32 64 us, 3.3 TB/s, bf16 71 us, 1.6 TB/s.
template <typename T, Mode MODE, int G>
__global__ void __launch_bounds__(1024) norm_kernel(const __grid_constant__ NormArgs a) {
    constexpr bool STAGED = MODE == kStaged, VEC = MODE != kApart;
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ RowSums sh;
    __shared__ uint64_t bars[kMostTeams * kMostStages];
    const uint32_t me = threadIdx.x, n = blockDim.x, stages = a.stages;
    const Weights<VEC> weights(reinterpret_cast<float*>(dyn), n * G);
    RowStages<T, 2> rows_in(dyn + n * G * 32, bars, a.cols, n * G * 8 * (uint32_t)sizeof(T), STAGED ? stages : 0, a.residual ? 2 : 1);
    grid_wait();
    grid_go();
    const uint64_t first = (uint64_t)blockIdx.x * blockDim.y + threadIdx.y, step = (uint64_t)gridDim.x * blockDim.y;
    const auto send = [&](uint32_t stage, uint64_t row) {
        const T* const from[2] = {static_cast<const T*>(a.x) + row * a.ldx, a.residual ? static_cast<const T*>(a.residual) + row * a.ldres : nullptr};
        rows_in.send(stage, from);
    };
    if (STAGED && me == 0)
        for (uint32_t i = 0; i < stages && first + i * step < a.rows; ++i) send(i, first + i * step);
    weights.fill(a.w, a.cols);
    __syncthreads();
    const uint32_t padded = (a.cols + 15) / 16 * 16;
    uint32_t half = 0;
    for (uint64_t row = first; row < a.rows + rows_ahead(); row += step, half ^= 1) {
        const bool live = MODE == kStaged || row < a.rows;
        Raw8<T> h[G];
        if constexpr (STAGED) {
            const uint32_t at = rows_in.take();
#pragma unroll
            for (int i = 0; i < G; ++i) {
                h[i] = load_staged<T>(at, me, n, i);
                if (a.residual) h[i] = rounded_sum<T>(h[i], load_staged<T>(at + rows_in.pitch, me, n, i));
            }
            if (!rows_in.ok) {
#pragma unroll
                for (int i = 0; i < G; ++i) h[i] = all_nan<T>();
            }
        } else {
#pragma unroll
            for (int i = 0; i < G; ++i) h[i] = load_direct<T, VEC>(static_cast<const T*>(a.x) + row * a.ldx, me, n, i, live ? a.cols : 0);
            if (a.residual) {
                Raw8<T> res[G];
#pragma unroll
                for (int i = 0; i < G; ++i) res[i] = load_direct<T, VEC>(static_cast<const T*>(a.residual) + row * a.ldres, me, n, i, live ? a.cols : 0);
#pragma unroll
                for (int i = 0; i < G; ++i) h[i] = rounded_sum<T>(h[i], res[i]);
            }
        }
        float2 sums = make_float2(0.f, 0.f);
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const Eight v = widen<T>(h[i]);
            if (a.q) {
                const Eight t = times(v, weights.get(me, n, i));
#pragma unroll
                for (int j = 0; j < 8; ++j) most = larger(most, t.at(j));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) sums = __ffma2_rn(v.v[j], v.v[j], sums);
        }
        float sum = __fadd_rn(sums.x, sums.y);
        uint32_t top = __float_as_uint(most);
        row_meet<true>(sh, half, sum, top);                // (all have read their part of the stage)
        if constexpr (STAGED) {
            if (me == 0 && row + stages * step < a.rows) send(rows_in.slot, row + stages * step);
            rows_in.next(stages);
        }
        if (MODE != kStaged && !live) continue;
        const float r = __frsqrt_rn(__fmaf_rn(sum, a.inv_cols, a.eps));
        if (me == 0 && a.r) a.r[row] = r;
        LineScale s = {};
        if (a.q) {
            s = line_scale(top);
            if (me == 0) a.scale[row] = __fmul_rn(s.scale, r);
        }
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const uint32_t c0 = column_of<VEC>(me, n, 8 * i);
            const Eight v = widen<T>(h[i]), w = weights.get(me, n, i);
            if (a.h) store_group<T, VEC>(static_cast<T*>(a.h) + row * a.ldh, me, n, i, a.cols, h[i]);
            if (a.y) store_group<T, VEC>(static_cast<T*>(a.y) + row * a.ldy, me, n, i, a.cols, narrow<T>(times(times(v, r), w)));
            if (a.q) {
                const uint2 code = codes_of(times(v, w), s.inv);
                int8_t* out = a.q + row * a.ldq;
                if constexpr (VEC) {
                    if (c0 < padded) *reinterpret_cast<uint2*>(out + c0) = code;
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (c0 + j * n < padded) out[c0 + j * n] = (int8_t)((j < 4 ? code.x : code.y) >> (8 * (j & 3)));
                }
            }
        }
    }
    if constexpr (STAGED) rows_in.leave(stages);
}

// Rows longer than a block holds: read twice, the second time from the caches (2048 x 20000 bf16 with a residual into codes: 150 us, 1.9 TB/s).  Where h is written it is what the second pass
// reads (it may have replaced an input).
template <typename T>
__global__ void __launch_bounds__(1024) norm_long_kernel(const __grid_constant__ NormArgs a) {
    __shared__ RowSums sh;
    grid_wait();
    grid_go();
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
        const float r = __frsqrt_rn(__fmaf_rn(sum, a.inv_cols, a.eps));
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
// With g = dy w: dx = r (g - h r^2 mean(g h)) + dres; dw = sum of dy h r over the rows.  A thread adds up dw of its columns over its
// team's rows, a block its teams', and leaves that in `part`; a second kernel adds the blocks' shares, always in the same order.
// 16384 x 4096 bf16 with dres: 91 to 94 us, 0.9 of the copy rate; 16384 x 1024: 40 us; 8192 x 4096 fp32: 95 us, 0.86; rows that start anywhere, 16384 x
// 1001: fp32 60 us, bf16 71.
// kStaged: a row is read from shared memory twice, before the meeting and after it, and its place is free once the team has met
// again.  (kApart with G = 4 has no room to keep it either.)
template <typename T, Mode MODE, int G>
__global__ void __launch_bounds__(512, MODE == kStaged ? 1 : 2) norm_grad_kernel(const __grid_constant__ NormGradArgs a) {
    constexpr bool STAGED = MODE == kStaged, VEC = MODE != kApart;
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ RowSums sh;
    __shared__ uint64_t bars[kMostTeams * kMostStages];
    const uint32_t me = threadIdx.x, n = blockDim.x, stages = a.stages;
    const Weights<VEC> weights(reinterpret_cast<float*>(dyn), n * G);
    RowStages<T, 3> rows_in(dyn + n * G * 32, bars, a.cols, n * G * 8 * (uint32_t)sizeof(T), STAGED ? stages : 0, a.arrays);
    grid_wait();
    grid_go();
    const uint64_t first = (uint64_t)blockIdx.x * blockDim.y + threadIdx.y, step = (uint64_t)gridDim.x * blockDim.y;
    const auto send = [&](uint32_t stage, uint64_t row) {
        const T* const from[3] = {static_cast<const T*>(a.dy) + row * a.lddy, static_cast<const T*>(a.h) + row * a.ldh,
                                  a.arrays == 3 ? static_cast<const T*>(a.dres) + row * a.lddres : nullptr};
        rows_in.send(stage, from);
    };
    if (STAGED && me == 0)
        for (uint32_t i = 0; i < stages && first + i * step < a.rows; ++i) send(i, first + i * step);
    weights.fill(a.w, a.cols);
    __syncthreads();
    Eight dw[G] = {};
    uint32_t half = 0, none = 0, filled = 0;               // filled: the stage whose row is done with
    for (uint64_t row = first; row < a.rows + rows_ahead(); row += step, half ^= 1) {
        const bool live = STAGED || row < a.rows;
        const uint32_t cols = live ? a.cols : 0;
        float r = live ? load_f32(a.r + row) : 0.f;
        const uint32_t at = STAGED ? rows_in.take() : 0;
        const T *pdy = static_cast<const T*>(a.dy) + row * a.lddy, *ph = static_cast<const T*>(a.h) + row * a.ldh;
        const T* pres = a.dres ? static_cast<const T*>(a.dres) + row * a.lddres : nullptr;
        if (STAGED && !rows_in.ok) r = CUDART_NAN_F;       // (a factor of every output)
        const auto get = [&](int which, const T* p, int i) {
            if constexpr (STAGED) return load_staged<T>(at + which * rows_in.pitch, me, n, i);
            else return load_direct<T, VEC>(p, me, n, i, cols);
        };
        constexpr bool kHeldOver = !STAGED && G <= 2;
        Raw8<T> dy[G], h[G];
        float2 dots = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < G; ++i) {
            dy[i] = get(0, pdy, i);
            h[i] = get(1, ph, i);
        }
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const Eight d = widen<T>(dy[i]), v = widen<T>(h[i]), g = times(d, weights.get(me, n, i)), z = times(v, r);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                dw[i].v[j] = __ffma2_rn(d.v[j], z.v[j], dw[i].v[j]);
                dots = __ffma2_rn(g.v[j], v.v[j], dots);
            }
        }
        float dot = __fadd_rn(dots.x, dots.y);
        row_meet<false>(sh, half, dot, none);              // (the row before this one has been read for the last time)
        if constexpr (STAGED) {
            if (stages > 1 && me == 0 && row != first && row + (stages - 1) * step < a.rows) send(filled, row + (stages - 1) * step);
            filled = rows_in.slot;
            rows_in.next(stages);
        }
        if (a.dx) {
            const float along = -__fmul_rn(__fmul_rn(__fmul_rn(r, r), a.inv_cols), dot);
#pragma unroll
            for (int i = 0; i < G; ++i) {
                const Eight g = times(widen<T>(kHeldOver ? dy[i] : get(0, pdy, i)), weights.get(me, n, i)), v = widen<T>(kHeldOver ? h[i] : get(1, ph, i));
                Eight e;
#pragma unroll
                for (int j = 0; j < 4; ++j) e.v[j] = __fmul2_rn(twice(r), __ffma2_rn(v.v[j], twice(along), g.v[j]));
                if (pres) e = plus(e, widen<T>(STAGED && a.arrays == 2 ? load_direct<T, true>(pres, me, n, i, cols) : get(2, pres, i)));
                store_group<T, VEC>(static_cast<T*>(a.dx) + row * a.lddx, me, n, i, cols, narrow<T>(e));
            }
        }
        if (STAGED && stages == 1) {                       // no row to spare: this one's place
            team_meet();
            if (me == 0 && row + step < a.rows) send(0, row + step);
        }
    }
    if constexpr (STAGED) rows_in.leave(stages);
    if (!a.part) return;
    float* out = a.part + (uint64_t)blockIdx.x * a.cols;
    if constexpr (STAGED) {
        // each team's sums where its rows were (whose places hold four bytes a column at least), in the weights' order; then added up.
        // The last row is read up to here by all of the team: it meets before its place is written.
        team_meet();
        const uint32_t held = n * G * 8, pitch = stages * a.arrays * held * (uint32_t)sizeof(T);
        unsigned char* rows = dyn + n * G * 32;
        float4* mine = reinterpret_cast<float4*>(rows + threadIdx.y * pitch);
#pragma unroll
        for (int i = 0; i < G; ++i) {
            mine[me + i * n] = make_float4(dw[i].v[0].x, dw[i].v[0].y, dw[i].v[1].x, dw[i].v[1].y);
            mine[n * G + me + i * n] = make_float4(dw[i].v[2].x, dw[i].v[2].y, dw[i].v[3].x, dw[i].v[3].y);
        }
        const bool failed = __syncthreads_or(!rows_in.ok);
        for (uint32_t c = threadIdx.y * n + me; c < a.cols; c += n * blockDim.y) {
            const uint32_t at = (c >> 2 & 1) * n * G * 4 + (c >> 3) * 4 + (c & 3);
            float sum = 0.f;
            for (uint32_t team = 0; team < blockDim.y; ++team) sum += reinterpret_cast<const float*>(rows + team * pitch)[at];
            out[c] = failed ? CUDART_NAN_F : sum;
        }
    } else {
        // a line a team, behind the weights; element j of thread t and group i at i 8 n + j n + t
        float* mine = reinterpret_cast<float*>(dyn) + (1 + threadIdx.y) * n * G * 8;
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) mine[(8 * i + j) * n + me] = dw[i].at(j);
        __syncthreads();
        for (uint32_t c = threadIdx.y * n + me; c < a.cols; c += n * blockDim.y) {
            const uint32_t g = c >> 3, at = VEC ? g / n * 8 * n + (c & 7) * n + g % n : c;
            float sum = 0.f;
            for (uint32_t team = 1; team <= blockDim.y; ++team) sum += reinterpret_cast<const float*>(dyn)[team * n * G * 8 + at];
            out[c] = sum;
        }
    }
}

// Rows longer than a block holds, dx: read twice (2048 x 20000 bf16 with dres and dw: 274 us, 1.2 TB/s; fp32 323).
template <typename T>
__global__ void __launch_bounds__(1024) norm_grad_long_kernel(const __grid_constant__ NormGradArgs a) {
    __shared__ RowSums sh;
    grid_wait();
    grid_go();
    uint32_t half = 0, none = 0;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, half ^= 1) {
        const T *pdy = static_cast<const T*>(a.dy) + row * a.lddy, *ph = static_cast<const T*>(a.h) + row * a.ldh;
        const T* pres = a.dres ? static_cast<const T*>(a.dres) + row * a.lddres : nullptr;
        const float r = load_f32(a.r + row);
        float dot = 0.f;
        for (uint32_t c = threadIdx.x; c < a.cols; c += 1024) dot = __fmaf_rn(__fmul_rn(load_one<T>(pdy + c), load_f32(a.w + c)), load_one<T>(ph + c), dot);
        row_meet<false>(sh, half, dot, none);
        const float along = __fmul_rn(__fmul_rn(__fmul_rn(r, r), a.inv_cols), dot);
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

// dw from the shares: 32 columns a block, 32 warps each a part of the shares.
__global__ void __launch_bounds__(1024) norm_sum_kernel(const float* part, uint32_t shares, uint64_t cols, float* dw) {
    __shared__ float sh[32][33];
    grid_wait();
    grid_go();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint64_t c = (uint64_t)blockIdx.x * 32 + lane;
    const uint32_t k0 = shares * warp / 32, k1 = shares * (warp + 1) / 32;
    float s = 0.f;
    if (c < cols) {
#pragma unroll 8
        for (uint32_t k = k0; k < k1; ++k) s += load_f32(part + k * cols + c);
    }
    sh[lane][warp] = s;
    __syncthreads();
    s = sh[warp][lane];                                    // column `warp`, share `lane`
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(kFullMask, s, d);
    if (lane == 0 && (uint64_t)blockIdx.x * 32 + warp < cols) dw[(uint64_t)blockIdx.x * 32 + warp] = s;
}

// ---- host ------------------------------------------------------------------------------------------
constexpr uint64_t kHeld = 16384;                          // columns that a team of 512 threads holds, 32 each
// How a launch is cut: how rows are read, groups of eight elements a thread, threads of a team and teams of a block, blocks an SM; kStaged:
// rows of a team under way and arrays among them.
struct NormShape {
    Mode mode;
    int groups;
    dim3 block;
    uint64_t per_sm;
    uint32_t stages, arrays;
};
constexpr uint64_t kMostSmem = 220 << 10;
// Rows that each find an SM's room for themselves: as many threads as groups.  In chains of launches (bf16, us, this way / the way of many rows):
//             codes with a residual           gradient with dres
//   columns   64 rows       296 rows          64 rows       296 rows
//   512       3.0 / 2.6     3.1 / 2.7         7.8 / 5.5     8.4 / 5.8
//   1536      2.6 / 3.5     2.9 / 3.6         5.8 / 6.0     7.1 / 6.3
//   4096      2.9 / 3.6     3.9 / 3.8         6.4 / 7.5     8.5 / 8.3
//   16384     5.5 / 5.9     8.6 / 8.7         15.2 / 15.1   27.8 / 20.1
// It is for the rows of a layer's width, one to a few a call; short ones, and gradients of more rows than SMs, lose by it.  At 444 rows it is
// slower at 4096 columns (5.5 / 5.0).
bool few_rows(uint64_t rows) { return rows <= 2 * 148; }

// Staged: of the cuts into `threads` threads that leave room for `least` rows a team, the one with the fewest instructions a row: a
// warp takes about 96 for a group of eight and 80 besides.  Returns false when none fits.
bool staged_shape(uint64_t cols, uint64_t element, uint32_t arrays, int groups, uint64_t threads, uint64_t per_sm, uint64_t least, NormShape& shape) {
    uint64_t lowest = ~0ull;
    for (int g = 1; g <= groups; g *= 2) {
        const uint64_t warps = (cols + 256 * g - 1) / (256 * g), n = warps * 32, held = n * g * 8, row = held * element * arrays;
        if (n > threads || kMostSmem / per_sm < held * 4 + least * row) continue;
        const uint64_t room = (kMostSmem / per_sm - held * 4) / row, teams = threads / n < room / least ? threads / n : room / least;
        const uint64_t cost = warps * (96 * g + 80) * (teams * n * 2 <= threads ? 2 : 1);         // (half a block idle: not for that)
        if (cost >= lowest) continue;
        lowest = cost;
        const uint64_t stages = room / teams;
        shape = {kStaged, g, dim3((unsigned)n, (unsigned)teams), per_sm, (uint32_t)(stages > kMostStages ? kMostStages : stages), arrays};
    }
    return lowest != ~0ull;
}
uint64_t shape_smem(const NormShape& s, uint64_t element, bool sums) {
    const uint64_t held = (uint64_t)s.block.x * s.groups * 8;
    return held * 4 + held * element * s.arrays * s.block.y * s.stages + (sums && s.mode != kStaged ? held * 4 * s.block.y : 0);
}
// Not staged: the fewest lanes that hold a short row, 32 elements each at most (single elements: eight); of a longer one few elements a
// thread, so that many loads are under way.
NormShape loose_shape(uint64_t cols, uint64_t threads, bool vec, int groups) {
    int g = 1;
    uint64_t n = 8;
    if (cols <= (vec ? 256ull * groups : 256)) {
        while (n < 32 && n * 8 < cols) n *= 2;
        while (n * 8 * g < cols) g *= 2;
    } else {
        while (cols > threads * 8 * g) g *= 2;
        n = (cols + 256 * g - 1) / (256 * g) * 32;
    }
    const uint64_t teams = n < 256 ? 256 / n : 1;
    return {vec ? kDirect : kApart, g, dim3((unsigned)n, (unsigned)(n > 32 && teams > 8 ? 8 : teams)), 1024 / (n * teams) > 0 ? 1024 / (n * teams) : 1, 0, 0};
}

// Blocks of the gradient at most, each with a share of dw: of a B200's SMs, not of the current device's, since the size of scratch
// follows from them.
uint64_t grad_shares(uint64_t rows, uint64_t cols) {
    const uint64_t most = cols > kHeld ? (rows + 63) / 64 : rows, cap = cols > kHeld ? 64 : 148 * 4;       // (long rows: 64 to a share at least)
    return most < cap ? most : cap;
}

// Whether rows start on 16-byte boundaries (`bytes` long: and end there).
bool row_fits(const void* p, uint64_t bytes, uint64_t rows, uint64_t stride) { return !p || (aligned(p, 16) && bytes % 16 == 0 && (rows == 1 || stride % 16 == 0)); }
template <typename K> cudaError_t allow_rows(K kernel, PerDevice<bool>& done) {
    const int slot = device_slot();
    if (slot >= 0 && done.v[slot]) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem);
    if (e == cudaSuccess && slot >= 0) done.v[slot] = true;
    return e;
}
// Calls f with a shape's mode and groups as types; the most groups that each mode is used with.
template <Mode MODE, int MOST, class F> cudaError_t with_groups(int groups, F&& f) {
    const std::integral_constant<Mode, MODE> mode;
    if (groups > MOST) return cudaErrorInvalidValue;       // (no shape asks for that)
    if constexpr (MOST == 4) {
        if (groups == 4) return f(mode, std::integral_constant<int, 4>());
    }
    return groups == 2 ? f(mode, std::integral_constant<int, 2>()) : f(mode, std::integral_constant<int, 1>());
}
template <int STAGED, int DIRECT, int APART, class F> cudaError_t with_shape(const NormShape& s, F&& f) {
    return s.mode == kStaged ? with_groups<kStaged, STAGED>(s.groups, f) : s.mode == kDirect ? with_groups<kDirect, DIRECT>(s.groups, f) : with_groups<kApart, APART>(s.groups, f);
}

template <typename T> cudaError_t launch_norm(NormArgs a, cudaStream_t st) {
    const uint64_t sms = (uint64_t)sm_count_now(), e = sizeof(T), bytes = a.cols * e;
    if (a.cols > kHeld) return launch_layer(norm_long_kernel<T>, (unsigned)(a.rows < 2 * sms ? a.rows : 2 * sms), 1024, 0, 1, st, a);
    const bool fits = row_fits(a.x, bytes, a.rows, a.ldx * e) && row_fits(a.residual, bytes, a.rows, a.ldres * e) && row_fits(a.h, bytes, a.rows, a.ldh * e) &&
                      row_fits(a.y, bytes, a.rows, a.ldy * e);
    const uint32_t arrays = a.residual ? 2 : 1;
    NormShape shape = loose_shape(a.cols, 1024, fits, 4);
    if (few_rows(a.rows)) shape.block.y = shape.block.x < 32 ? 32 / shape.block.x : 1;
    else if (fits && a.cols > 1024 && !staged_shape(a.cols, e, arrays, 2, 512, 2, 1, shape)) (void)staged_shape(a.cols, e, arrays, 2, 1024, 1, 1, shape);
    a.stages = shape.stages;
    const uint64_t want = (a.rows + shape.block.y - 1) / shape.block.y, most = shape.per_sm * sms;
    return with_shape<2, 4, 2>(shape, [&](auto mode, auto g) {
        static PerDevice<bool> done;
        const auto kernel = norm_kernel<T, decltype(mode)::value, decltype(g)::value>;
        const cudaError_t err = allow_rows(kernel, done);
        if (err != cudaSuccess) return err;
        return launch_layer(kernel, (unsigned)(want < most ? want : most), shape.block, shape_smem(shape, e, false), 1, st, a);
    });
}

template <typename T> cudaError_t launch_norm_grad(NormGradArgs a, float* dw, cudaStream_t st) {
    const uint64_t sms = (uint64_t)sm_count_now(), e = sizeof(T), bytes = a.cols * e;
    uint64_t shares = grad_shares(a.rows, a.cols);
    cudaError_t err = cudaSuccess;
    if (a.cols > kHeld) {
        // dw first: dx may take the place of dy
        if (dw) err = launch_layer(norm_grad_long_dw_kernel<T>, dim3((a.cols + 255) / 256, (unsigned)shares), 256, 0, 1, st, a);
        if (err == cudaSuccess && a.dx) err = launch_layer(norm_grad_long_kernel<T>, (unsigned)(a.rows < 2 * sms ? a.rows : 2 * sms), 1024, 0, 1, st, a);
    } else {
        const bool fits = row_fits(a.dy, bytes, a.rows, a.lddy * e) && row_fits(a.h, bytes, a.rows, a.ldh * e) && row_fits(a.dres, bytes, a.rows, a.lddres * e) &&
                          row_fits(a.dx, bytes, a.rows, a.lddx * e);
        NormShape shape = loose_shape(a.cols, 512, fits, 2);
        if (few_rows(a.rows)) {
            shape.block.y = shape.block.x < 32 ? 32 / shape.block.x : 1;
            if (shape.mode == kDirect && shape.groups == 4) {
                shape.mode = kStaged;                      // (what G = 4 would read twice stays on chip)
                shape.stages = 1;
                shape.arrays = 2;
            }
        } else if (fits && a.cols > 1024) {
            // (dres straight from memory where its rows do not fit too; at the widest, one row at a time)
            if (!staged_shape(a.cols, e, a.dres ? 3 : 2, 4, 512, 1, 2, shape) && !staged_shape(a.cols, e, 2, 4, 512, 1, 2, shape)) (void)staged_shape(a.cols, e, 2, 4, 512, 1, 1, shape);
        }
        a.stages = shape.stages;
        a.arrays = shape.arrays;
        const uint64_t want = (a.rows + shape.block.y - 1) / shape.block.y, most = shape.per_sm * 148 < shares ? shape.per_sm * 148 : shares;
        shares = want < most ? want : most;
        err = with_shape<4, 2, 4>(shape, [&](auto mode, auto g) {
            static PerDevice<bool> done;
            const auto kernel = norm_grad_kernel<T, decltype(mode)::value, decltype(g)::value>;
            const cudaError_t allowed = allow_rows(kernel, done);
            if (allowed != cudaSuccess) return allowed;
            return launch_layer(kernel, (unsigned)shares, shape.block, shape_smem(shape, e, true), 1, st, a);
        });
    }
    if (err != cudaSuccess || !dw) return err;
    return launch_layer(norm_sum_kernel, (unsigned)((a.cols + 31) / 32), 1024, 0, 1, st, a.part, (uint32_t)shares, (uint64_t)a.cols, dw);
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
    const NormArgs a{x_dev, residual_dev, w_dev, h_dev, y_dev, q_dev, scale_dev, r_dev, rows, ldx, ldres, ldh, ldy, ldq, (uint32_t)cols, 0, eps, 1.0f / (float)cols};
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
                         rows, lddy, ldh, lddres, lddx, (uint32_t)cols, 0, 2, 1.0f / (float)cols};
    return layer_status(with_type(type, [&](auto t) { return launch_norm_grad<decltype(t)>(a, dw_dev, st); }));
}

}  // extern "C"
