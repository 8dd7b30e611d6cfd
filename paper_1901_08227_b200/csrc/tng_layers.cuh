// Building blocks of the training-layer operators (8-bit linear layers, dropout): element types,
// 8-wide loads and stores, and the Philox counters they draw from.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tng_device.cuh"
#include "tng_internal.h"

namespace tng {

// Third counter word = layer + tag.  Gradient coding uses the worker index (< 64) there, so layers and
// gradient coding never share a counter under one key; nor do rounding and dropout of one layer.
constexpr uint32_t kTagRounding = 1u << 30, kTagDropout = 1u << 31;

// What a kernel needs of a tng_draw: the round keys and the counter words that a launch shares, and what follows from
// them alone in the first round.  Of the 20 wide multiplies of a call two depend only on these and on the row, and
// one more only on the column, where neighbouring calls differ by a constant: see DrawRow and draw_words.
struct DrawArgs {
    uint32_t rk[20];
    uint32_t row0, step_key;       // step ^ second key of round 1
    uint32_t hi_key, lo;           // word2's product of round 1: high word ^ first key, low word ^ first key of round 2
};
inline DrawArgs make_draw(const tng_draw& d, uint32_t tag) {
    DrawArgs a;
    philox_round_keys(d.seed_lo, d.seed_hi, a.rk);
    a.row0 = (uint32_t)d.row0;
    a.step_key = d.step ^ a.rk[1];
    const uint64_t p = (uint64_t)kPhiloxMul1 * (d.layer + tag);
    a.hi_key = (uint32_t)(p >> 32) ^ a.rk[0];
    a.lo = (uint32_t)p ^ a.rk[2];
    return a;
}
// Host checks shared by the calls that take a draw over `rows` rows.
inline bool draw_ok(const tng_draw* d, uint64_t rows) {
    return d->layer < (1u << 30) && d->row0 <= (1ull << 32) && rows <= (1ull << 32) - d->row0;
}

// The row's share of rounds 1 and 2.
struct DrawRow {
    uint32_t hi_key, lo;           // M0 * (round 1's first word): high word ^ second key of round 2, low word
};
__device__ __forceinline__ DrawRow draw_row(const DrawArgs& a, uint32_t row) {
    const uint64_t p = static_cast<uint64_t>(kPhiloxMul0) * (a.hi_key ^ (a.row0 + row));
    return {static_cast<uint32_t>(p >> 32) ^ a.rk[3], static_cast<uint32_t>(p)};
}
// M0 * col4, what the column brings to round 1; the next column group's is this + M0.
__device__ __forceinline__ uint64_t draw_column(uint32_t col4) { return static_cast<uint64_t>(kPhiloxMul0) * col4; }
// The four words of columns 4*col4 .. 4*col4+3 of a row (row counted from the draw's row0).
__device__ __forceinline__ uint4 draw_words(const DrawArgs& a, const DrawRow& r, uint64_t column) {
    // after round 1: (hi_key ^ row, lo, hi(column) ^ step_key, lo(column)); round 2 from that
    const uint64_t p = static_cast<uint64_t>(kPhiloxMul1) * (static_cast<uint32_t>(column >> 32) ^ a.step_key);
    uint32_t c0 = static_cast<uint32_t>(p >> 32) ^ a.lo, c1 = static_cast<uint32_t>(p);
    uint32_t c2 = r.hi_key ^ static_cast<uint32_t>(column), c3 = r.lo;
#pragma unroll
    for (int round = 2; round < 10; ++round) {
        const uint64_t p0 = static_cast<uint64_t>(kPhiloxMul0) * c0;
        const uint64_t p1 = static_cast<uint64_t>(kPhiloxMul1) * c2;
        const uint32_t n0 = static_cast<uint32_t>(p1 >> 32) ^ c1 ^ a.rk[2 * round];
        const uint32_t n2 = static_cast<uint32_t>(p0 >> 32) ^ c3 ^ a.rk[2 * round + 1];
        c1 = static_cast<uint32_t>(p1);
        c3 = static_cast<uint32_t>(p0);
        c0 = n0;
        c2 = n2;
    }
    return make_uint4(c0, c1, c2, c3);
}

// The layer kernels are launched so that one may be set up while the one before it on the stream ends (a few
// microseconds a launch, in chains of short kernels).  Every thread calls grid_wait() before it touches global memory:
// it returns when all earlier work on the stream is complete and visible; grid_go() lets the next launch begin its set-up.
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_go() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Loads of what an earlier launch may have written.  Not the read-only path (__ldg, or a const __restrict__ parameter): that
// one is for data that nobody writes while the kernel exists, and here the launch before may still be writing when
// this one starts to wait; volatile, so that none moves ahead of grid_wait().
__device__ __forceinline__ uint4 load16(const void* p) {
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint4 load16_once(const void* p) {              // read once: first to leave the caches
    uint4 v;
    asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t load4_bits(const void* p) {
    uint32_t v;
    asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t load2_bits(const void* p) {
    uint16_t v;
    asm volatile("ld.global.u16 %0, [%1];" : "=h"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ float load_f32(const float* p) { return __uint_as_float(load4_bits(p)); }

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32(float v) { return v; }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32(float v) { return __float2half_rn(v); }

// Two 16-bit values packed in a word, first one in the low half.
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Eight consecutive elements as they lie in memory: 16 bytes of a 16-bit type, 32 of fp32.
template <typename T> struct Raw8 {
    uint4 w[sizeof(T) / 2];
};
template <typename T> __device__ __forceinline__ Raw8<T> load_raw8(const T* p) {   // p 16-byte aligned
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.w[i] = load16(reinterpret_cast<const uint4*>(p) + i);
    return r;
}
template <typename T> __device__ __forceinline__ void widen8(const Raw8<T>& r, float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        v[0] = __uint_as_float(r.w[0].x); v[1] = __uint_as_float(r.w[0].y);
        v[2] = __uint_as_float(r.w[0].z); v[3] = __uint_as_float(r.w[0].w);
        v[4] = __uint_as_float(r.w[1].x); v[5] = __uint_as_float(r.w[1].y);
        v[6] = __uint_as_float(r.w[1].z); v[7] = __uint_as_float(r.w[1].w);
    } else {
        float2 a = unpack2<T>(r.w[0].x); v[0] = a.x; v[1] = a.y;
        a = unpack2<T>(r.w[0].y); v[2] = a.x; v[3] = a.y;
        a = unpack2<T>(r.w[0].z); v[4] = a.x; v[5] = a.y;
        a = unpack2<T>(r.w[0].w); v[6] = a.x; v[7] = a.y;
    }
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&v)[8]) {   // p 16-byte aligned
    uint4* o = reinterpret_cast<uint4*>(p);
    if constexpr (sizeof(T) == 4) {
        o[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        o[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    } else {
        o[0] = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
    }
}

__device__ __forceinline__ bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <typename... P, typename... A>
cudaError_t launch_layer(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, unsigned cluster, cudaStream_t st, const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

// What a call returns for the last step of its work.  The runtime remembers an error until it is asked for, and calls that
// ask after their launch would take it for their own: it is cleared here.
inline tng_status layer_status(cudaError_t e) {
    if (e == cudaSuccess) return TNG_OK;
    (void)cudaGetLastError();
    return TNG_ERR_CUDA;
}
// Calls f(T()) for the element type of `type`.
template <class F> inline cudaError_t with_type(tng_dtype type, F&& f) {
    switch (type) {
        case TNG_F32: return f(float());
        case TNG_BF16: return f(__nv_bfloat16());
        case TNG_F16: return f(__half());
    }
    return cudaErrorInvalidValue;
}
inline size_t type_bytes(tng_dtype t) { return t == TNG_F32 ? 4 : 2; }
inline bool type_ok(tng_dtype t) { return t == TNG_F32 || t == TNG_BF16 || t == TNG_F16; }
// Sizes and row pointers of an activation matrix and of codes.
inline bool dims_ok(uint64_t rows, uint64_t cols) { return rows < (1ull << 31) && cols < (1ull << 31); }
inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool matrix_ok(const void* p, tng_dtype t, uint64_t cols, uint64_t ld) {
    return p && aligned(p, type_bytes(t)) && ld >= cols && ld < (1ull << 32);
}
inline bool codes_ok(const void* p, uint64_t cols, uint64_t ld) {
    return p && aligned(p, 16) && ld >= cols && ld % 16 == 0 && ld < (1ull << 32);
}

}  // namespace tng
