// Products of 8-bit codes with scales for each row of either side:
//   out[i][j] = (float(sum_l a[i][l] b[j][l]) sa[i]) sb[j] + bias[j].
#include "tng_layers.cuh"

namespace tng {
namespace {

__device__ __forceinline__ float scaled(int acc, float sa, float sb, float bias) {
    return __fadd_rn(__fmul_rn(__fmul_rn((float)acc, sa), sb), bias);
}

// Four codes starting at l, zero beyond k (l is a multiple of 4, rows are padded to 16 bytes).
__device__ __forceinline__ int word4(const int8_t* row, uint64_t l, uint64_t k) {
    if (l >= k) return 0;
    uint32_t w = *reinterpret_cast<const uint32_t*>(row + l);
    if (l + 4 > k) w &= (1u << (8 * (k - l))) - 1u;
    return (int)w;
}

// 64 x 64 outputs a CTA, 4 x 4 a thread, 64 codes of the contraction at a time.
template <typename T>
__global__ void __launch_bounds__(256) product8_tile_kernel(Product8 p) {
    __shared__ int sa[16][65], sb[16][65];
    const uint64_t i0 = (uint64_t)blockIdx.y * 64, j0 = (uint64_t)blockIdx.x * 64;
    const uint32_t tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    int acc[4][4] = {};
    for (uint64_t l0 = 0; l0 < p.k; l0 += 64) {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const uint32_t r = ty + 16 * h;
            sa[tx][r] = i0 + r < p.m ? word4(p.a + (i0 + r) * p.lda, l0 + 4 * tx, p.k) : 0;
            sb[tx][r] = j0 + r < p.n ? word4(p.b + (j0 + r) * p.ldb, l0 + 4 * tx, p.k) : 0;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 16; ++w)
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
                for (int x = 0; x < 4; ++x) acc[y][x] = __dp4a(sa[w][ty * 4 + y], sb[w][tx * 4 + x], acc[y][x]);
        __syncthreads();
    }
    for (int y = 0; y < 4; ++y)
        for (int x = 0; x < 4; ++x) {
            const uint64_t i = i0 + ty * 4 + y, j = j0 + tx * 4 + x;
            if (i < p.m && j < p.n)
                static_cast<T*>(p.out)[i * p.ldo + j] = from_f32<T>(scaled(acc[y][x], p.sa[i], p.sb[j], p.bias ? p.bias[j] : 0.f));
        }
}

}  // namespace

cudaError_t launch_product8(const Product8& p, cudaStream_t st) {
    const uint64_t gx = (p.n + 63) / 64, gy = (p.m + 63) / 64;
    if (gy > 65535) return cudaErrorInvalidValue;
    return with_type(p.type, [&](auto t) {
        product8_tile_kernel<decltype(t)><<<dim3((unsigned)gx, (unsigned)gy), 256, 0, st>>>(p);
        return cudaGetLastError();
    });
}

}  // namespace tng

using namespace tng;

extern "C" tng_status tng_product8(const int8_t* a_dev, uint64_t lda, const float* sa_dev, const int8_t* b_dev, uint64_t ldb,
                                   const float* sb_dev, const float* bias_dev, uint64_t m, uint64_t n, uint64_t k, void* out_dev,
                                   tng_dtype type, uint64_t ldo, void* stream) {
    if (!type_ok(type) || n < 1 || k < 1 || k > TNG_MAX_CONTRACTION || !dims_ok(m, n)) return TNG_ERR_INVALID_ARG;
    if (m == 0) return TNG_OK;
    if (!codes_ok(a_dev, k, lda) || !codes_ok(b_dev, k, ldb) || !sa_dev || !sb_dev || !aligned(sa_dev, 4) || !aligned(sb_dev, 4) ||
        !aligned(bias_dev, 4) || !matrix_ok(out_dev, type, n, ldo))
        return TNG_ERR_INVALID_ARG;
    const Product8 p{a_dev, b_dev, lda, ldb, sa_dev, sb_dev, bias_dev, m, n, k, out_dev, type, ldo};
    return launch_product8(p, static_cast<cudaStream_t>(stream)) == cudaSuccess ? TNG_OK : TNG_ERR_CUDA;
}
