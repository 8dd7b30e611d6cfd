// Rows of a table by token, and the table's gradient.
//
//   y[t] = table[ids[t]] scale;  dtable[v] = scale * (sum of dy[t] over the t with ids[t] = v, t ascending)
//
// Both are bound by memory, the gradient by writing the whole table (4 bytes an element, a worker's row of gradients has no
// other way to say zero) and reading dy once.  Its sums are formed in an order that the ids alone decide: the places are
// sorted by id (a stable sort, so that equal ids stay in order), cut into chunks of equal length, and a run of equal ids that crosses
// chunks is summed from its chunks' parts in order.  No atomic addition, and a token that half the batch shares costs no more
// than any other.
#include "tng_layers.cuh"
#include "tng_umma.cuh"

namespace tng {
namespace {

template <typename I> __device__ __forceinline__ int64_t load_id(const void* ids, uint64_t t) {
    I v;
    if constexpr (sizeof(I) == 8) asm volatile("ld.global.u64 %0, [%1];" : "=l"(v) : "l"(static_cast<const I*>(ids) + t));
    else asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(static_cast<const I*>(ids) + t));
    return v;
}
template <typename T> __device__ __forceinline__ float load_element(const T* p) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(load4_bits(p));
    else return unpack2<T>(load2_bits(p)).x;
}

// ---- lookup ------------------------------------------------------------------------------------------
struct EmbedArgs {
    const void *table, *ids;
    void* y;
    uint64_t vocab, ldt, tokens, ldy;
    uint32_t width, segments;      // segments of kSegment elements a row
    float scale;
};
constexpr int kEmbedThreads = 128;
constexpr uint32_t kSegment = kEmbedThreads * 8;

// A block takes segments of rows in turn: eight elements a thread, neighbours where rows start on 16-byte boundaries (VEC),
// else 128 apart.
template <typename S, typename T, typename I, bool VEC>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const __grid_constant__ EmbedArgs a) {
    grid_wait();
    grid_go();
    const uint64_t units = a.tokens * a.segments;
    for (uint64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const uint64_t t = u / a.segments;
        const uint32_t first = (uint32_t)(u - t * a.segments) * kSegment;
        const int64_t id = load_id<I>(a.ids, t);
        const bool in = id >= 0 && (uint64_t)id < a.vocab;
        const S* src = static_cast<const S*>(a.table) + (in ? (uint64_t)id : 0) * a.ldt;
        T* dst = static_cast<T*>(a.y) + t * a.ldy;
        const float blank = id == -1 ? 0.f : __int_as_float(0x7FFFFFFF);
        const uint32_t c0 = VEC ? first + threadIdx.x * 8 : first + threadIdx.x;
        float v[8];
        if (VEC && c0 + 8 <= a.width) {
            if (in) widen8(load_raw8(src + c0), v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = in ? __fmul_rn(v[j], a.scale) : blank;
            store8(dst + c0, v);
        } else {
            const uint32_t step = VEC ? 1 : kEmbedThreads;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = in && c0 + j * step < a.width ? load_element<S>(src + c0 + j * step) : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + j * step < a.width) dst[c0 + j * step] = from_f32<T>(in ? __fmul_rn(v[j], a.scale) : blank);
        }
    }
}

// ---- gradient: the places sorted by id ------------------------------------------------------------------
// One cluster of eight CTAs sorts, least significant digits first, up to nine bits a pass (two passes up to 262143 ids): each warp
// owns consecutive places, counts its digits, and after the cluster has exchanged the CTAs' counts moves its places in order.  Places
// without an id sort behind all others.  The cluster's other CTAs (every further cluster of the launch) meanwhile write zeros
// to the rows that no place names; each finds its own from a bitmap of its rows, for which it looks through all ids.
constexpr int kSortThreads = 1024, kSortCtas = 8, kDigits = 512;
struct SortArgs {
    const void* ids;
    uint64_t tokens, vocab, ldd;
    uint32_t *key[2], *place[2];   // what the passes go between; the last one ends in [0]
    float* dtable;
    uint32_t width, passes, bits, per_fill;   // per_fill: rows of the table to a filling CTA, at most kFillRows
};
constexpr uint32_t kFillRows = kDigits * 32 * 32;          // a bit each of the counters' space
constexpr uint32_t kSortSmem = 32 * kDigits * 4;

template <typename I>
__global__ void __launch_bounds__(kSortThreads, 1) embed_sort_kernel(const __grid_constant__ SortArgs a) {
    extern __shared__ uint32_t counts[];                   // [warp][digit]
    __shared__ uint32_t total[kDigits], warp_sum[32];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    grid_wait();
    grid_go();
    if (blockIdx.x >= kSortCtas) {                         // ---- fill
        const uint64_t r0 = (uint64_t)(blockIdx.x - kSortCtas) * a.per_fill;
        const uint32_t rows = r0 >= a.vocab ? 0u : a.vocab - r0 < a.per_fill ? (uint32_t)(a.vocab - r0) : a.per_fill;
        for (uint32_t i = threadIdx.x; i < (rows + 31) / 32; i += kSortThreads) counts[i] = 0;
        __syncthreads();
        if (rows) {
#pragma unroll 4
            for (uint64_t t = threadIdx.x; t < a.tokens; t += kSortThreads) {
                const uint64_t at = (uint64_t)load_id<I>(a.ids, t) - r0;
                if (at < rows) atomicOr(&counts[at >> 5], 1u << (at & 31));
            }
        }
        __syncthreads();
        const bool vec = (reinterpret_cast<uintptr_t>(a.dtable) | a.ldd * 4) % 16 == 0;
        for (uint32_t r = warp; r < rows; r += 32) {
            if (counts[r >> 5] >> (r & 31) & 1u) continue;
            float* dst = a.dtable + (r0 + r) * a.ldd;
            uint32_t c = lane;
            if (vec) {
                for (uint32_t g = lane; g < a.width / 4; g += 32) reinterpret_cast<float4*>(dst)[g] = make_float4(0.f, 0.f, 0.f, 0.f);
                c += a.width / 4 * 4;
            }
            for (; c < a.width; c += 32) dst[c] = 0.f;
        }
        return;
    }
    // ---- sort
    const uint32_t cta = cluster_rank();
    const uint64_t mine0 = a.tokens * cta / kSortCtas, mine1 = a.tokens * (cta + 1) / kSortCtas;
    const uint64_t from = mine0 + (mine1 - mine0) * warp / 32, to = mine0 + (mine1 - mine0) * (warp + 1) / 32;
    const uint32_t digits = 1u << a.bits;
    for (uint32_t p = 0; p < a.passes; ++p) {
        const uint32_t shift = p * a.bits;
        const uint32_t in = (a.passes - p) & 1u, out = in ^ 1u;            // the last pass writes [0]
        const auto key_at = [&](uint64_t t) {
            if (p > 0) return __ldcg(a.key[in] + t);
            const uint64_t id = (uint64_t)load_id<I>(a.ids, t);
            return id < a.vocab ? (uint32_t)id : (uint32_t)a.vocab;
        };
        uint32_t* own = counts + warp * kDigits;
        for (uint32_t d = lane; d < digits; d += 32) own[d] = 0;
        __syncwarp();
        for (uint64_t t = from + lane; t < to; t += 32) atomicAdd(&own[(key_at(t) >> shift) & (digits - 1)], 1u);
        __syncthreads();
        // counts of the CTA, the warps' turned into offsets within them
        const uint32_t d = threadIdx.x;
        if (d < digits) {
            uint32_t s = 0;
#pragma unroll 8
            for (uint32_t w = 0; w < 32; ++w) {
                const uint32_t n = counts[w * kDigits + d];
                counts[w * kDigits + d] = s;
                s += n;
            }
            total[d] = s;
        }
        cluster_sync_all();
        // where the CTA's places with digit d go: behind all with a lower digit, and those of the CTAs before with the same one
        uint32_t before = 0, all = 0;
        if (d < digits) {
            uint32_t v[kSortCtas];
#pragma unroll
            for (uint32_t c = 0; c < kSortCtas; ++c) v[c] = (uint32_t)cluster_ld(cluster_map(smem_u32(&total[d]), c));
#pragma unroll
            for (uint32_t c = 0; c < kSortCtas; ++c) {
                if (c < cta) before += v[c];
                all += v[c];
            }
        }
        uint32_t scan = all;
#pragma unroll
        for (int i = 1; i < 32; i <<= 1) {
            const uint32_t o = __shfl_up_sync(kFullMask, scan, i);
            if (lane >= (uint32_t)i) scan += o;
        }
        if (lane == 31) warp_sum[warp] = scan;
        __syncthreads();
        uint32_t lower = lane < warp ? warp_sum[lane] : 0u;
        lower = __reduce_add_sync(kFullMask, lower);
        const uint32_t base = lower + scan - all + before;
        if (d < digits) {
#pragma unroll 8
            for (uint32_t w = 0; w < 32; ++w) counts[w * kDigits + d] += base;
        }
        __syncthreads();
        for (uint64_t t0 = from; t0 < to; t0 += 32) {
            const uint64_t t = t0 + lane;
            const bool live = t < to;
            const uint32_t key = live ? key_at(t) : 0u, digit = live ? (key >> shift) & (digits - 1) : digits;
            const uint32_t place = p > 0 && live ? __ldcg(a.place[in] + t) : (uint32_t)t;
            const uint32_t same = __match_any_sync(kFullMask, digit);
            const uint32_t rank = __popc(same & ((1u << lane) - 1)), leader = __ffs(same) - 1;
            uint32_t at = 0;
            if (live && lane == leader) {
                at = own[digit];
                own[digit] = at + __popc(same);
            }
            __syncwarp();
            at = __shfl_sync(kFullMask, at, leader) + rank;
            if (live) {
                __stcg(a.key[out] + at, key);
                __stcg(a.place[out] + at, place);
            }
        }
        cluster_sync_all();                                // the next pass reads what the other CTAs moved
    }
}

// ---- gradient: sums over the runs ------------------------------------------------------------------------
// A block has a chunk of the sorted places and 8 columns a thread.  Runs that lie within the chunk are done; of a run that
// comes in from the chunk before, the part goes to line 2 c of `part`, of one that goes on into the next chunk to line 2 c + 1 (a
// run that does both: 2 c).
struct GradArgs {
    const void* dy;
    const uint32_t *key, *place;
    float *part, *dtable;
    uint64_t tokens, vocab, lddy, ldd;
    uint32_t width, chunk, chunks;
    float scale;
};
constexpr int kGradThreads = 128;
constexpr uint32_t kGradSpan = kGradThreads * 8;

template <bool VEC> __device__ __forceinline__ uint32_t span_column(uint32_t j) {
    return blockIdx.y * kGradSpan + (VEC ? threadIdx.x * 8 + j : threadIdx.x + j * kGradThreads);
}
template <bool VEC> __device__ __forceinline__ void put_sums(float* dst, uint32_t width, const float (&v)[8]) {
    const uint32_t c0 = span_column<VEC>(0);
    if (VEC && c0 + 8 <= width && aligned16(dst)) {
        store8(dst + c0, v);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (span_column<VEC>(j) < width) dst[span_column<VEC>(j)] = v[j];
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kGradThreads) embed_sum_kernel(const __grid_constant__ GradArgs a) {
    grid_wait();
    grid_go();
    const uint64_t s = (uint64_t)blockIdx.x * a.chunk, e = s + a.chunk < a.tokens ? s + a.chunk : a.tokens;
    const uint32_t c0 = span_column<VEC>(0);
    const bool whole = VEC && c0 + 8 <= a.width;
    float sum[8] = {};
    uint32_t run = load4_bits(a.key + s);
    bool from_before = s > 0 && load4_bits(a.key + s - 1) == run;
    const auto leave = [&](bool goes_on) {
        if (run < a.vocab) {
            if (from_before || goes_on) {
                put_sums<VEC>(a.part + (2ull * blockIdx.x + (from_before ? 0 : 1)) * a.width, a.width, sum);
            } else {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(sum[j], a.scale);
                put_sums<VEC>(a.dtable + run * a.ldd, a.width, v);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.f;
        from_before = false;
    };
    constexpr int kAhead = 4;
    for (uint64_t i = s; i < e; i += kAhead) {
        uint32_t key[kAhead];
        float v[kAhead][8];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            key[u] = i + u < e ? load4_bits(a.key + i + u) : 0u;
            const T* row = static_cast<const T*>(a.dy) + (uint64_t)(i + u < e ? load4_bits(a.place + i + u) : 0u) * a.lddy;
            const bool live = i + u < e && key[u] < a.vocab;
            if (whole) {
                widen8(live ? load_raw8(row + c0) : Raw8<T>{}, v[u]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[u][j] = live && span_column<VEC>(j) < a.width ? load_element<T>(row + span_column<VEC>(j)) : 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u >= e) break;
            if (key[u] != run) {
                leave(false);
                run = key[u];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += v[u][j];
        }
    }
    leave(e < a.tokens && load4_bits(a.key + e) == run);
}

// A run that goes on beyond the chunk it begins in: its parts, chunk by chunk.
__global__ void __launch_bounds__(kGradThreads) embed_join_kernel(const __grid_constant__ GradArgs a) {
    __shared__ uint32_t last;
    grid_wait();
    grid_go();
    const uint32_t c = blockIdx.x;                         // (never the last chunk)
    const uint64_t s = (uint64_t)c * a.chunk, e = s + a.chunk;
    const uint32_t run = load4_bits(a.key + e - 1);
    if (run >= a.vocab || load4_bits(a.key + e) != run) return;             // (uniform over the block)
    if (s > 0 && load4_bits(a.key + s) == run && load4_bits(a.key + s - 1) == run) return;   // it began before this chunk
    // the first chunk after c that the run does not come in from
    if (threadIdx.x == 0) last = a.chunks;
    __syncthreads();
    for (uint32_t j = c + 1; j < a.chunks; j += kGradThreads) {
        const uint32_t k = j + threadIdx.x;
        const bool ends = k < a.chunks && (load4_bits(a.key + (uint64_t)k * a.chunk) != run);
        if (ends) atomicMin(&last, k);
        if (__syncthreads_or(ends)) break;
    }
    const uint32_t end = last;
    float sum[8];
    const auto part = [&](uint64_t line, int j) {
        const uint32_t col = span_column<false>(j);
        return col < a.width ? load_f32(a.part + line * a.width + col) : 0.f;
    };
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = part(2ull * c + 1, j);
#pragma unroll 4
    for (uint32_t k = c + 1; k < end; ++k) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += part(2ull * k, j);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = __fmul_rn(sum[j], a.scale);
    put_sums<false>(a.dtable + run * a.ldd, a.width, sum);
}

// ---- host ------------------------------------------------------------------------------------------
// Places to a chunk: 32, more for long batches, so that the runs' parts stay a small share of the traffic and few enough to join.
uint64_t chunk_of(uint64_t tokens) {
    uint64_t c = 32;
    while (tokens / c > 4096) c *= 2;
    return c;
}
uint64_t up256(uint64_t n) { return (n + 255) / 256 * 256; }

template <typename S, typename T> cudaError_t launch_embed(const EmbedArgs& a, bool wide_ids, cudaStream_t st) {
    const bool vec = aligned(a.table, 16) && a.ldt * sizeof(S) % 16 == 0 && aligned(a.y, 16) && (a.tokens == 1 || a.ldy * sizeof(T) % 16 == 0);
    const uint64_t units = a.tokens * a.segments, cap = (uint64_t)sm_count_now() * 16;
    const auto kernel = wide_ids ? (vec ? embed_kernel<S, T, int64_t, true> : embed_kernel<S, T, int64_t, false>)
                                 : (vec ? embed_kernel<S, T, int32_t, true> : embed_kernel<S, T, int32_t, false>);
    return launch_layer(kernel, (unsigned)(units < cap ? units : cap), kEmbedThreads, 0, 1, st, a);
}

}  // namespace
}  // namespace tng

using namespace tng;

extern "C" {

tng_status tng_embed(const void* table_dev, tng_dtype table_type, uint64_t vocab, uint64_t width, uint64_t ldt, const void* ids_dev,
                     uint32_t id_bytes, uint64_t tokens, float scale, void* y_dev, tng_dtype type, uint64_t ldy, void* stream) {
    if (!type_ok(table_type) || !type_ok(type) || width < 1 || vocab < 1 || !dims_ok(tokens, width) || !dims_ok(vocab, width) ||
        (id_bytes != 4 && id_bytes != 8))
        return TNG_ERR_INVALID_ARG;
    if (tokens == 0) return TNG_OK;
    if (!matrix_ok(table_dev, table_type, width, ldt) || !matrix_ok(y_dev, type, width, ldy) || !ids_dev || !aligned(ids_dev, id_bytes)) return TNG_ERR_INVALID_ARG;
    const EmbedArgs a{table_dev, ids_dev, y_dev, vocab, ldt, tokens, ldy, (uint32_t)width, (uint32_t)((width + kSegment - 1) / kSegment), scale};
    return layer_status(with_type(table_type, [&](auto s) {
        return with_type(type, [&](auto t) { return launch_embed<decltype(s), decltype(t)>(a, id_bytes == 8, static_cast<cudaStream_t>(stream)); });
    }));
}

size_t tng_embed_grad_scratch_bytes(uint64_t tokens, uint64_t width) {
    if (tokens == 0) return 256;
    const uint64_t chunk = chunk_of(tokens), chunks = (tokens + chunk - 1) / chunk;
    return (size_t)(4 * up256(tokens * 4) + up256(chunks * 2 * width * 4));
}

tng_status tng_embed_grad(const void* dy_dev, tng_dtype type, uint64_t tokens, uint64_t width, uint64_t lddy, const void* ids_dev,
                          uint32_t id_bytes, uint64_t vocab, float scale, float* dtable_dev, uint64_t ldd, void* scratch_dev, void* stream) {
    if (!type_ok(type) || width < 1 || vocab < 1 || !dims_ok(tokens, width) || !dims_ok(vocab, width) || (id_bytes != 4 && id_bytes != 8) ||
        !matrix_ok(dtable_dev, TNG_F32, width, ldd))
        return TNG_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (tokens == 0) return layer_status(cudaMemset2DAsync(dtable_dev, ldd * 4, 0, width * 4, vocab, st));
    if (!matrix_ok(dy_dev, type, width, lddy) || !ids_dev || !aligned(ids_dev, id_bytes) || !scratch_dev || !aligned(scratch_dev, 256)) return TNG_ERR_INVALID_ARG;
    unsigned char* at = static_cast<unsigned char*>(scratch_dev);
    SortArgs s = {};
    s.ids = ids_dev; s.tokens = tokens; s.vocab = vocab; s.ldd = ldd; s.dtable = dtable_dev; s.width = (uint32_t)width;
    const uint64_t list = up256(tokens * 4);
    for (int i = 0; i < 2; ++i) {
        s.key[i] = reinterpret_cast<uint32_t*>(at + 2 * i * list);
        s.place[i] = reinterpret_cast<uint32_t*>(at + (2 * i + 1) * list);
    }
    uint32_t bits = 1;
    while (vocab >> bits) ++bits;                          // of the largest key, vocab itself
    s.passes = (bits + 8) / 9;
    s.bits = (bits + s.passes - 1) / s.passes;
    const uint64_t clusters = (uint64_t)sm_count_now() / kSortCtas, fills = (clusters > 2 ? clusters - 1 : 1) * kSortCtas;
    uint64_t per = (vocab + fills - 1) / fills;
    if (per > kFillRows) per = kFillRows;
    s.per_fill = (uint32_t)per;
    const uint64_t ctas = ((vocab + per - 1) / per + kSortCtas - 1) / kSortCtas * kSortCtas + kSortCtas;
    static PerDevice<bool> done[2];
    const bool wide = id_bytes == 8;
    const auto sort = wide ? embed_sort_kernel<int64_t> : embed_sort_kernel<int32_t>;
    const int slot = device_slot();
    cudaError_t e = cudaSuccess;
    if (slot < 0 || !done[wide].v[slot]) {
        e = cudaFuncSetAttribute(sort, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSortSmem);
        if (e == cudaSuccess && slot >= 0) done[wide].v[slot] = true;
    }
    if (e == cudaSuccess) e = launch_layer(sort, (unsigned)ctas, kSortThreads, kSortSmem, kSortCtas, st, s);
    if (e != cudaSuccess) return layer_status(e);
    const uint64_t chunk = chunk_of(tokens), chunks = (tokens + chunk - 1) / chunk, spans = (width + kGradSpan - 1) / kGradSpan;
    if (spans > 65535) return TNG_ERR_INVALID_ARG;
    const GradArgs g{dy_dev, s.key[0], s.place[0], reinterpret_cast<float*>(at + 4 * list), dtable_dev, tokens, vocab, lddy, ldd,
                     (uint32_t)width, (uint32_t)chunk, (uint32_t)chunks, scale};
    const dim3 grid((unsigned)chunks, (unsigned)spans);
    e = with_type(type, [&](auto t) {
        using T = decltype(t);
        const bool vec = aligned(dy_dev, 16) && (tokens == 1 || lddy * sizeof(T) % 16 == 0);
        return launch_layer(vec ? embed_sum_kernel<T, true> : embed_sum_kernel<T, false>, grid, kGradThreads, 0, 1, st, g);
    });
    if (e == cudaSuccess && chunks > 1) e = launch_layer(embed_join_kernel, dim3((unsigned)chunks - 1, (unsigned)spans), kGradThreads, 0, 1, st, g);
    return layer_status(e);
}

}  // extern "C"
