// Linear layers with 8-bit products: quantisers and products composed, forward and backward.
#include "tng_layers.cuh"

using namespace tng;

namespace {

uint64_t up256(uint64_t n) { return (n + 255) / 256 * 256; }
// Codes of `lines` lines of `n` values and their scales, each part on a 256-byte boundary.
uint64_t codes_bytes(uint64_t lines, uint64_t n) { return up256(lines * tng_code_stride(n)); }
uint64_t scales_bytes(uint64_t lines) { return up256(4 * lines); }

struct Carver {
    unsigned char* at;
    template <typename T> T* take(uint64_t bytes) {
        T* p = reinterpret_cast<T*>(at);
        at += bytes;
        return p;
    }
};

}  // namespace

extern "C" {

size_t tng_linear8_scratch_bytes(uint64_t tokens, uint64_t k) {
    return product8_codes_tokens(tokens, k) ? 0 : (size_t)(codes_bytes(tokens, k) + scales_bytes(tokens));
}

tng_status tng_linear8(const void* x_dev, tng_dtype type, uint64_t tokens, uint64_t k, uint64_t ldx, const int8_t* w_dev,
                       uint64_t ldw, const float* sw_dev, uint64_t n, const float* bias_dev, void* y_dev, uint64_t ldy,
                       void* scratch_dev, void* stream) {
    if (!type_ok(type) || n < 1 || k < 1 || k > TNG_MAX_CONTRACTION || !dims_ok(tokens, n)) return TNG_ERR_INVALID_ARG;
    if (tokens == 0) return TNG_OK;
    if (!matrix_ok(x_dev, type, k, ldx) || !codes_ok(w_dev, k, ldw) || !sw_dev || !aligned(sw_dev, 4) || !aligned(bias_dev, 4) ||
        !matrix_ok(y_dev, type, n, ldy))
        return TNG_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (product8_codes_tokens(tokens, k)) {
        const Product8 p{nullptr, w_dev, 0, ldw, nullptr, sw_dev, bias_dev, tokens, n, k, y_dev, type, ldy};
        return layer_status(launch_linear8_stream(x_dev, ldx, p, st));
    }
    if (!scratch_dev || !aligned(scratch_dev, 256)) return TNG_ERR_INVALID_ARG;
    Carver c{static_cast<unsigned char*>(scratch_dev)};
    int8_t* q = c.take<int8_t>(codes_bytes(tokens, k));
    float* s = c.take<float>(scales_bytes(tokens));
    const uint64_t ldq = tng_code_stride(k);
    const cudaError_t e = launch_quant8_rows(x_dev, type, tokens, k, ldx, nullptr, q, ldq, s, st);
    if (e != cudaSuccess) return layer_status(e);
    const Product8 p{q, w_dev, ldq, ldw, s, sw_dev, bias_dev, tokens, n, k, y_dev, type, ldy};
    return layer_status(launch_product8(p, st));
}

size_t tng_linear8_grad_scratch_bytes(uint64_t tokens, uint64_t k, uint64_t n) {
    if (tokens == 0) return 256;
    return (size_t)(codes_bytes(tokens, n) + scales_bytes(tokens) + codes_bytes(n, tokens) + scales_bytes(n) + codes_bytes(k, tokens) +
                    scales_bytes(k) + up256(4 * (k + tokens + quant8_cols_scratch(tokens, n))));
}

tng_status tng_linear8_grad(const void* dy_dev, uint64_t lddy, const void* x_dev, uint64_t ldx, tng_dtype type, uint64_t tokens,
                            uint64_t k, uint64_t n, const int8_t* wt_dev, uint64_t ldwt, const float* swt_dev, const tng_draw* draw,
                            void* dx_dev, uint64_t lddx, float* dw_dev, uint64_t lddw, float* db_dev, void* scratch_dev, void* stream) {
    if (!type_ok(type) || n < 1 || k < 1 || !dims_ok(tokens, n) || !dims_ok(tokens, k) || (draw && !draw_ok(draw, tokens)))
        return TNG_ERR_INVALID_ARG;
    if ((dx_dev && n > TNG_MAX_CONTRACTION) || (dw_dev && tokens > TNG_MAX_CONTRACTION)) return TNG_ERR_INVALID_ARG;
    if ((dw_dev && !matrix_ok(dw_dev, TNG_F32, k, lddw)) || !aligned(db_dev, 4)) return TNG_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (tokens == 0) {                             // an empty batch has zero gradients
        cudaError_t e = dw_dev ? cudaMemset2DAsync(dw_dev, lddw * 4, 0, k * 4, n, st) : cudaSuccess;
        if (e == cudaSuccess && db_dev) e = cudaMemsetAsync(db_dev, 0, n * 4, st);
        return layer_status(e);
    }
    if (!matrix_ok(dy_dev, type, n, lddy) || !scratch_dev || !aligned(scratch_dev, 256)) return TNG_ERR_INVALID_ARG;
    if (dw_dev && !matrix_ok(x_dev, type, k, ldx)) return TNG_ERR_INVALID_ARG;
    if (dx_dev && (!matrix_ok(dx_dev, type, k, lddx) || !codes_ok(wt_dev, n, ldwt) || !swt_dev || !aligned(swt_dev, 4)))
        return TNG_ERR_INVALID_ARG;
    // With a sum over the tokens to form, dy's row and column codes come from the same passes, and x's columns share their
    // launches: clear the maxima (side by side), maxima, codes, products.  dx alone needs the rows only.
    Carver c{static_cast<unsigned char*>(scratch_dev)};
    const uint64_t ldr = tng_code_stride(n), ldc = tng_code_stride(tokens);
    int8_t* qr = c.take<int8_t>(codes_bytes(tokens, n));
    float* sr = c.take<float>(scales_bytes(tokens));
    int8_t* qy = c.take<int8_t>(codes_bytes(n, tokens));
    float* sy = c.take<float>(scales_bytes(n));
    int8_t* qx = c.take<int8_t>(codes_bytes(k, tokens));
    float* sx = c.take<float>(scales_bytes(k));
    uint32_t* tops_x = c.take<uint32_t>(0);
    uint32_t* tops_rows = tops_x + k;
    uint32_t* work_y = tops_rows + tokens;
    cudaError_t e = cudaSuccess;
    if (dw_dev || db_dev) {
        e = cudaMemsetAsync(tops_x, 0, (k + tokens + n) * 4, st);
        const Quant8Cols jobs[2] = {{dy_dev, tokens, n, lddy, draw, qy, ldc, sy, db_dev, work_y, dx_dev ? tops_rows : nullptr, dx_dev ? qr : nullptr, ldr, sr},
                                    {x_dev, tokens, k, ldx, nullptr, qx, ldc, sx, nullptr, tops_x, nullptr, nullptr, 0, nullptr}};
        if (e == cudaSuccess) e = launch_quant8_cols(jobs, dw_dev ? 2 : 1, type, st);
    } else if (dx_dev) {
        e = launch_quant8_rows(dy_dev, type, tokens, n, lddy, draw, qr, ldr, sr, st);
    }
    if (e != cudaSuccess) return layer_status(e);
    const Product8 to_x{qr, wt_dev, ldr, ldwt, sr, swt_dev, nullptr, tokens, k, n, dx_dev, type, lddx};
    const Product8 to_w{qy, qx, ldc, ldc, sy, sx, nullptr, n, k, tokens, dw_dev, TNG_F32, lddw};
    e = dx_dev && dw_dev ? launch_product8_two(to_x, to_w, st) : dx_dev ? launch_product8(to_x, st) : dw_dev ? launch_product8(to_w, st) : cudaSuccess;
    return layer_status(e);
}

}  // extern "C"
