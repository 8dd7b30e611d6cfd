// How a value becomes an 8-bit code: shared by the quantisers and by the product that codes its tokens itself.
#pragma once

#include "tng_layers.cuh"

namespace tng {

constexpr uint32_t kInfBits = 0x7F800000u;
constexpr float kTiny = 0x1p-120f;

struct LineScale {
    float scale, inv;    // inv = 0: all codes of the line are zero
};
// `bits`: largest |x| of the line as a bit pattern; a NaN's is above every number's and wins.
__device__ __forceinline__ LineScale line_scale(uint32_t bits) {
    const float top = __uint_as_float(bits);
    LineScale s;
    s.scale = __fdiv_rn(top, 127.f);
    s.inv = __fdiv_rn(127.f, top);
    if (top < kTiny) s.scale = s.inv = 0.f;
    if (bits >= kInfBits) s.inv = 0.f;
    return s;
}

// Adding 1.5 * 2^23 leaves the rounded integer in the low bits: to nearest even with round-to-nearest, the
// floor with round-down; the low byte is the two's complement code.
template <bool DRAW> __device__ __forceinline__ uint32_t code_bits(float x, float inv, uint32_t word) {
    const float v = __fmul_rn(x, inv);
    if constexpr (DRAW) {
        // cut before the floor: -127 <= t < 128 gives the same codes as cutting the floor to [-127, 127]
        const float t = fminf(fmaxf(__fmaf_rn(__uint2float_rn(word >> 8), 0x1p-24f, v), -127.f), 127.5f);   // v + u, u exact
        return __float_as_uint(__fadd_rd(t, 12582912.f));
    } else {
        return __float_as_uint(__fadd_rn(v, 12582912.f));
    }
}
__device__ __forceinline__ uint32_t pack_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

// Eight codes of a row; a line with inv = 0 has code zero everywhere (0 * NaN would not).
template <bool DRAW> __device__ __forceinline__ uint2 code8(const float (&v)[8], float inv, const DrawArgs& d, const DrawRow& r, uint32_t group) {
    uint32_t w[8] = {};
    if constexpr (DRAW) {
        const uint64_t column = draw_column(2 * group);
        const uint4 a = draw_words(d, r, column), b = draw_words(d, r, column + kPhiloxMul0);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    }
    uint32_t q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = code_bits<DRAW>(v[j], inv, w[j]);
    return inv == 0.f ? make_uint2(0u, 0u) : make_uint2(pack_bytes(q[0], q[1], q[2], q[3]), pack_bytes(q[4], q[5], q[6], q[7]));
}

// Eight elements of a row from column c as they lie in memory; zero beyond the row.  VEC: the row is 16-byte aligned.
template <typename T, bool VEC> __device__ __forceinline__ Raw8<T> fetch_raw8(const T* row, uint64_t c, uint64_t cols) {
    if (VEC && c + 8 <= cols) return load_raw8(row + c);
    Raw8<T> r;
    uint32_t* w = reinterpret_cast<uint32_t*>(&r);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = c + j < cols ? load4_bits(row + c + j) : 0u;
    } else {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(row) + c;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = c + 2 * j < cols ? load2_bits(h + 2 * j) : 0u, hi = c + 2 * j + 1 < cols ? load2_bits(h + 2 * j + 1) : 0u;
            w[j] = lo | hi << 16;
        }
    }
    return r;
}
template <typename T> __device__ __forceinline__ Raw8<T> zero_raw8() {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.w[i] = make_uint4(0u, 0u, 0u, 0u);
    return r;
}

// Running maximum of magnitudes as integers, which order like the magnitudes with NaN on top: 16-bit types two to a word.
template <typename T> __device__ __forceinline__ uint32_t top_word(uint32_t w, uint32_t m) {
    if constexpr (sizeof(T) == 4) return max(m, w & 0x7FFFFFFFu);
    else return __vmaxu2(m, w & 0x7FFF7FFFu);
}
template <typename T> __device__ __forceinline__ uint32_t top_raw8(const Raw8<T>& r, uint32_t m) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) m = top_word<T>(r.w[i].x, top_word<T>(r.w[i].y, top_word<T>(r.w[i].z, top_word<T>(r.w[i].w, m))));
    return m;
}
// A magnitude (the low half of a word for 16-bit types) as the bit pattern of the fp32 value.
template <typename T> __device__ __forceinline__ uint32_t top_bits(uint32_t m) {
    if constexpr (sizeof(T) == 4) return m;
    else return __float_as_uint(unpack2<T>(m).x);
}
template <typename T> __device__ __forceinline__ uint32_t top_of_halves(uint32_t m) {
    if constexpr (sizeof(T) == 4) return m;
    else return max(m & 0xFFFFu, m >> 16);
}

}  // namespace tng
