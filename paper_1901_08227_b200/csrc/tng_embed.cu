// Rows of a table by token, and the table's gradient.
//
//   y[t] = table[ids[t]] scale;  dtable[v] = scale * (sum of dy[t] over the t with ids[t] = v, t ascending)
//
// Both are bound by memory, the gradient by writing the whole table (4 bytes an element, a worker's row of gradients has no
// other way to say zero) and reading dy once.  Its sums are formed in an order that the ids alone decide: the places are
// sorted by id (a stable sort, so that equal ids stay in order), cut into chunks of equal length, and a run of equal ids that crosses
// chunks is summed from its chunks' parts in order.  No atomic addition, and a token that half the batch shares costs no more
// than any other.
#include "tng_codes.cuh"
#include "tng_umma.cuh"

namespace tng {
namespace {

template <typename I> __device__ __forceinline__ int64_t load_id(const void* ids, uint64_t t) {
    I v;
    if constexpr (sizeof(I) == 8) asm volatile("ld.global.u64 %0, [%1];" : "=l"(v) : "l"(static_cast<const I*>(ids) + t));
    else asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(static_cast<const I*>(ids) + t));
    return v;
}
__device__ __forceinline__ uint2 load_pair(const uint2* p) {
    uint2 v;
    asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
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

// Bound by memory; 16384 of 65536 rows of 2048, fp32 to bf16: 22 us; of 2047, which start anywhere: 33.  A block takes segments of rows in turn: eight elements a thread, neighbours where rows start on 16-byte boundaries (VEC),
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
// One cluster sorts, least significant digits first, up to nine bits a pass (two passes up to 262143 ids): each warp owns consecutive
// places, counts its digits, and after the cluster's CTAs have exchanged their counts moves its places in order.  Places without an
// id sort behind all others.  (A cluster of four: all of the launch's clusters have to run at once, and those of eight leave 20 SMs
// out.)  CTAS = 1 (up to kSmallTokens places): the lists stay in shared memory between the passes, and nothing is exchanged.  The launch's other CTAs meanwhile write zeros to the rows that no place names;
// each finds its own from a bitmap of its rows, for which it looks through all ids.  The zeros leave as bulk copies, a row each.
constexpr int kSortThreads = 1024, kDigits = 512;
constexpr uint32_t kSmallTokens = 8192;
struct SortArgs {
    const void* ids;
    uint64_t tokens, vocab, ldd;
    uint2* pair[2];                // (id, place): what the passes go between; the last one ends in [0]
    uint32_t* crossing;            // counter of embed_sum_kernel, cleared here
    float* dtable;
    uint32_t width, passes, bits, fills;       // fills: the CTAs that fill take every so manieth row
};
constexpr uint32_t kFillRows = kDigits * 32 * 32;          // a bit each of the counters' space
constexpr uint32_t kCountBytes = 32 * kDigits * 4, kZeroBytes = 16384;
template <int CTAS> constexpr uint32_t kSortSmem = kCountBytes + (CTAS == 1 ? 2 * 8 * kSmallTokens : kZeroBytes);

// Zeros into this CTA's rows (part, part + fills, ...) that no id names: together the CTAs sweep the table from its beginning to its end,
// which memory takes faster than a part of the table each (65536 x 2048: 124 us), and frequent ids, low as a rule, are spread.
template <typename I> __device__ __forceinline__ void fill_rows(const SortArgs& a, uint32_t part, uint32_t* bits, unsigned char* zeros) {
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t vocab = (uint32_t)a.vocab, rows = part < vocab ? (vocab - part - 1) / a.fills + 1 : 0u;
    for (uint32_t i = threadIdx.x; i < (rows + 31) / 32; i += kSortThreads) bits[i] = 0;
    for (uint32_t i = threadIdx.x; i < kZeroBytes / 16; i += kSortThreads) reinterpret_cast<uint4*>(zeros)[i] = make_uint4(0u, 0u, 0u, 0u);
    smem_to_copies();
    __syncthreads();
    if (!rows) return;
    for (uint64_t t0 = threadIdx.x; t0 < a.tokens; t0 += 8 * kSortThreads) {
        uint64_t id[8];                                    // eight loads under way
#pragma unroll
        for (int i = 0; i < 8; ++i) id[i] = t0 + i * kSortThreads < a.tokens ? (uint64_t)load_id<I>(a.ids, t0 + i * kSortThreads) : ~0ull;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t at = (uint32_t)id[i] / a.fills;
            if (id[i] < vocab && (uint32_t)id[i] - at * a.fills == part) atomicOr(&bits[at >> 5], 1u << (at & 31));
        }
    }
    __syncthreads();
    const bool vec = (reinterpret_cast<uintptr_t>(a.dtable) | a.ldd * 4) % 16 == 0;
    const uint32_t whole = vec ? a.width / 4 * 16 : 0;     // bytes of a row that go as copies
    for (uint32_t r = warp; r < rows; r += 32) {
        if (bits[r >> 5] >> (r & 31) & 1u) continue;
        float* dst = a.dtable + (part + (uint64_t)r * a.fills) * a.ldd;
        if (lane == 0)
            for (uint32_t at = 0; at < whole; at += kZeroBytes) bulk_store(reinterpret_cast<unsigned char*>(dst) + at, smem_u32(zeros), whole - at < kZeroBytes ? whole - at : kZeroBytes);
        for (uint32_t c = whole / 4 + lane; c < a.width; c += 32) dst[c] = 0.f;
    }
    if (lane == 0) tile_store_wait_all();
}

template <typename I, int CTAS>
__global__ void __launch_bounds__(kSortThreads, 1) embed_sort_kernel(const __grid_constant__ SortArgs a) {
    extern __shared__ __align__(16) uint32_t counts[];     // [warp][digit], then the lists or the zeros
    __shared__ uint32_t total[kDigits], warp_sum[32];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint2* lists = reinterpret_cast<uint2*>(counts + 32 * kDigits);
    grid_wait();
    grid_go();
    if (blockIdx.x >= CTAS) {
        fill_rows<I>(a, blockIdx.x - CTAS, counts, reinterpret_cast<unsigned char*>(lists));
        return;
    }
    const uint32_t cta = CTAS > 1 ? cluster_rank() : 0u;
    if (cta == 0 && threadIdx.x == 0) *a.crossing = 0;
    const uint64_t mine0 = a.tokens * cta / CTAS, mine1 = a.tokens * (cta + 1) / CTAS;
    const uint64_t from = mine0 + (mine1 - mine0) * warp / 32, to = mine0 + (mine1 - mine0) * (warp + 1) / 32;
    const uint32_t digits = 1u << a.bits;
    // A warp's keys come in batches of kBatch loads under way at once; a single batch (kept) serves the counting and the moving.
    constexpr int kBatch = 8;
    const bool single = to - from <= 32 * kBatch;
    for (uint32_t p = 0; p < a.passes; ++p) {
        const uint32_t shift = p * a.bits;
        const uint32_t in = (a.passes - p) & 1u, out = in ^ 1u;            // the last pass writes [0]
        uint32_t key[kBatch], place[kBatch];
        const auto load = [&](uint64_t t0) {
            if (p > 0) {
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    const uint64_t t = t0 + 32 * i + lane;
                    const uint2 v = t < to ? CTAS > 1 ? __ldcg(a.pair[in] + t) : lists[in * kSmallTokens + t] : make_uint2(0u, 0u);
                    key[i] = v.x;
                    place[i] = v.y;
                }
            } else {
                uint64_t id[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) id[i] = t0 + 32 * i + lane < to ? (uint64_t)load_id<I>(a.ids, t0 + 32 * i + lane) : 0u;
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    key[i] = id[i] < a.vocab ? (uint32_t)id[i] : (uint32_t)a.vocab;
                    place[i] = (uint32_t)t0 + 32 * i + lane;
                }
            }
        };
        uint32_t* own = counts + warp * kDigits;
        for (uint32_t d = lane; d < digits; d += 32) own[d] = 0;
        __syncwarp();
        uint32_t same[kBatch];
        // lanes with a digit alike, bit by bit (a warp-wide match takes longer: 32768 places 40 us, so 34)
        const auto match = [&](uint64_t t0) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i) same[i] = __ballot_sync(kFullMask, t0 + 32 * i + lane < to);
            for (uint32_t bit = shift; bit < shift + a.bits; ++bit) {
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    const uint32_t ones = __ballot_sync(kFullMask, key[i] >> bit & 1u);
                    same[i] &= key[i] >> bit & 1u ? ones : ~ones;
                }
            }
        };
        // the place of batch i's key among those of its digit, and the digit's counter moved on
        const auto claim = [&](uint64_t t0, int i) -> uint32_t {
            const bool live = t0 + 32 * i + lane < to;
            const uint32_t digit = (key[i] >> shift) & (digits - 1), leader = live ? __ffs(same[i]) - 1 : 0;
            uint32_t at = 0;
            if (live && lane == leader) {
                at = own[digit];
                own[digit] = at + __popc(same[i]);
            }
            __syncwarp();
            return __shfl_sync(kFullMask, at, leader) + __popc(same[i] & ((1u << lane) - 1));
        };
        for (uint64_t t0 = from; t0 < to; t0 += 32 * kBatch) {
            load(t0);
            match(t0);
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (t0 + 32 * i < to) (void)claim(t0, i);
        }
        __syncthreads();
        // counts of the CTA, the warps' turned into offsets within them
        const uint32_t d = threadIdx.x;
        uint32_t all = 0, before = 0;
        if (d < digits) {
#pragma unroll 8
            for (uint32_t w = 0; w < 32; ++w) {
                const uint32_t n = counts[w * kDigits + d];
                counts[w * kDigits + d] = all;
                all += n;
            }
        }
        if constexpr (CTAS > 1) {
            if (d < digits) total[d] = all;
            cluster_sync_all();
            // where the CTA's places with digit d go: behind all with a lower digit, and those of the CTAs before with the same one
            if (d < digits) {
                uint32_t v[CTAS];
#pragma unroll
                for (uint32_t c = 0; c < CTAS; ++c) v[c] = (uint32_t)cluster_ld(cluster_map(smem_u32(&total[d]), c));
                all = 0;
#pragma unroll
                for (uint32_t c = 0; c < CTAS; ++c) {
                    if (c < cta) before += v[c];
                    all += v[c];
                }
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
        for (uint64_t t0 = from; t0 < to; t0 += 32 * kBatch) {
            if (!single) {
                load(t0);
                match(t0);
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                if (t0 + 32 * i >= to) break;
                const uint32_t at = claim(t0, i);
                if (t0 + 32 * i + lane >= to) continue;
                if (CTAS > 1 || p + 1 == a.passes) __stcg(a.pair[out] + at, make_uint2(key[i], place[i]));
                else lists[out * kSmallTokens + at] = make_uint2(key[i], place[i]);
            }
        }
        if (CTAS > 1) cluster_sync_all();                  // the next pass reads what the other CTAs moved
        else __syncthreads();
    }
}

// ---- gradient: sums over the runs ------------------------------------------------------------------------
// A block has a chunk of the sorted places and 8 columns a thread.  Runs that lie within the chunk are done; of a run that
// comes in from the chunk before, the part goes to line 2 c of `part`, of one that goes on into the next chunk to line 2 c + 1 (a
// run that does both: 2 c).  Chunks from which a run goes on that began there are listed for embed_join_kernel.
// 32768 x 2048 bf16: 38 us, 4.6 TB/s of what it reads and writes.
struct GradArgs {
    const void* dy;
    const uint2* pair;
    uint32_t *crossing, *list;     // how many chunks are listed, and which, in any order
    float *part, *dtable;
    uint64_t tokens, vocab, lddy, ldd;
    uint32_t width, chunk, chunks;
    float scale;
};
constexpr int kGradThreads = 128;
constexpr uint32_t kGradSpan = kGradThreads * 8, kGradList = 128;

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
    __shared__ uint32_t keys[kGradList], places[kGradList];
    grid_wait();
    grid_go();
    const uint64_t s = (uint64_t)blockIdx.x * a.chunk, e = s + a.chunk < a.tokens ? s + a.chunk : a.tokens;
    const uint32_t c0 = span_column<VEC>(0);
    const bool whole = VEC && c0 + 8 <= a.width;
    float sum[8] = {};
    uint32_t run = load4_bits(a.pair + s);
    bool from_before = s > 0 && load4_bits(a.pair + s - 1) == run;
    const auto leave = [&](bool goes_on) {
        if (run < a.vocab) {
            if (from_before || goes_on) {
                put_sums<VEC>(a.part + (2ull * blockIdx.x + (from_before ? 0 : 1)) * a.width, a.width, sum);
                if (!from_before && blockIdx.y == 0 && threadIdx.x == 0) a.list[atomicAdd(a.crossing, 1u)] = blockIdx.x;
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
    constexpr int kAhead = sizeof(T) == 2 ? 8 : 4;          // rows under way
    for (uint64_t i0 = s; i0 < e; i0 += kGradList) {
        const uint32_t n = e - i0 < kGradList ? (uint32_t)(e - i0) : kGradList;
        __syncthreads();
        if (threadIdx.x < n) {
            const uint2 v = load_pair(a.pair + i0 + threadIdx.x);
            keys[threadIdx.x] = v.x;
            places[threadIdx.x] = v.y;
        }
        __syncthreads();
#pragma unroll 1
        for (uint32_t i = 0; i < n; i += kAhead) {
            Raw8<T> v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const bool live = i + u < n && keys[i + u] < a.vocab;
                const T* row = static_cast<const T*>(a.dy) + (uint64_t)(live ? places[i + u] : 0u) * a.lddy;
                v[u] = zero_raw8<T>();
                if (whole) {
                    if (live) v[u] = load_raw8(row + c0);
                } else {
                    uint32_t* w = reinterpret_cast<uint32_t*>(&v[u]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t c = span_column<VEC>(j);
                        if constexpr (sizeof(T) == 4) w[j] = live && c < a.width ? load4_bits(row + c) : 0u;
                        else w[j / 2] |= (live && c < a.width ? load2_bits(row + c) : 0u) << (16 * (j & 1));
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (i + u >= n) break;
                if (keys[i + u] != run) {
                    leave(false);
                    run = keys[i + u];
                }
                float f[8];
                widen8(v[u], f);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += f[j];
            }
        }
    }
    leave(e < a.tokens && load4_bits(a.pair + e) == run);
}

// The listed runs, from their parts chunk by chunk: a block has 512 columns of one, eight warps each a share of the chunks.  (Latency: five
// dependent loads a run.)
constexpr int kJoinThreads = 256, kJoinHeld = 16;
constexpr uint32_t kJoinSpan = 32 * kJoinHeld;
__global__ void __launch_bounds__(kJoinThreads) embed_join_kernel(const __grid_constant__ GradArgs a) {
    __shared__ uint32_t last;
    __shared__ float sums[8][kJoinSpan];
    grid_wait();
    grid_go();
    const uint32_t spans = (a.width + kJoinSpan - 1) / kJoinSpan, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint64_t units = (uint64_t)load4_bits(a.crossing) * spans;
    for (uint64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const uint32_t c = load4_bits(a.list + u / spans), c0 = (uint32_t)(u % spans) * kJoinSpan + lane;
        const uint32_t run = load4_bits(a.pair + (uint64_t)(c + 1) * a.chunk);
        // the first chunk after c + 1 that the run does not come in from
        if (threadIdx.x == 0) last = a.chunks;
        __syncthreads();
        for (uint32_t j = c + 2; j < a.chunks; j += kJoinThreads) {
            const uint32_t k = j + threadIdx.x;
            const bool ends = k < a.chunks && load4_bits(a.pair + (uint64_t)k * a.chunk) != run;
            if (ends) atomicMin(&last, k);
            if (__syncthreads_or(ends)) break;
        }
        __syncthreads();
        const uint32_t n = last - c;                       // parts: line 2 c + 1, then the lines 2 k of the chunks after c
        const uint32_t k0 = (uint32_t)((uint64_t)n * warp / 8), k1 = (uint32_t)((uint64_t)n * (warp + 1) / 8);
        float sum[kJoinHeld] = {};
        for (uint32_t k = k0; k < k1; k += 2) {
            float v[2][kJoinHeld];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float* line = a.part + (k + i == 0 ? 2ull * c + 1 : 2ull * (c + k + i)) * a.width;
#pragma unroll
                for (int j = 0; j < kJoinHeld; ++j) v[i][j] = k + i < k1 && c0 + 32 * j < a.width ? load_f32(line + c0 + 32 * j) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < kJoinHeld; ++j) sum[j] += v[i][j];
        }
#pragma unroll
        for (int j = 0; j < kJoinHeld; ++j) sums[warp][lane + 32 * j] = sum[j];
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < kJoinSpan; i += kJoinThreads) {
            const uint32_t col = (uint32_t)(u % spans) * kJoinSpan + i;
            float t = 0.f;
#pragma unroll
            for (int w = 0; w < 8; ++w) t += sums[w][i];
            if (col < a.width) a.dtable[run * a.ldd + col] = __fmul_rn(t, a.scale);
        }
        __syncthreads();
    }
}

// ---- host ------------------------------------------------------------------------------------------
// Places to a chunk: 32; fewer where that leaves SMs idle, more for long batches, so that the runs' parts stay few enough to join.
uint64_t chunk_of(uint64_t tokens) {
    uint64_t c = 4;
    while (c < 32 && tokens / c > 4 * 148) c *= 2;
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

// The sorting cluster and, on the other SMs, the CTAs that fill.
template <typename I, int CTAS> cudaError_t launch_sort(SortArgs s, cudaStream_t st) {
    static PerDevice<bool> done;
    static PerDevice<int> resident;                        // CTAs of the launch that run at once
    const auto kernel = embed_sort_kernel<I, CTAS>;
    const int slot = device_slot();
    if (slot < 0 || !done.v[slot]) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSortSmem<CTAS>);
        if (e != cudaSuccess) return e;
        if (slot >= 0) done.v[slot] = true;
    }
    uint64_t most = slot >= 0 ? (uint64_t)resident.v[slot] : 0;
    if (!most) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(CTAS);
        cfg.blockDim = dim3(kSortThreads);
        cfg.dynamicSmemBytes = kSortSmem<CTAS>;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = CTAS;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int n = 0;
        if (CTAS == 1) n = sm_count_now();
        else if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) (void)cudaGetLastError();
        most = (uint64_t)(n > 2 ? n : 2) * CTAS;
        if (slot >= 0) resident.v[slot] = (int)most;
    }
    uint64_t fills = most - CTAS;
    while (s.vocab > fills * kFillRows) fills *= 2;        // (rows of a CTA: a bit each)
    if (fills > s.vocab) fills = (s.vocab + CTAS - 1) / CTAS * CTAS;
    s.fills = (uint32_t)fills;
    const uint64_t ctas = fills + CTAS;
    return launch_layer(kernel, (unsigned)ctas, kSortThreads, kSortSmem<CTAS>, CTAS, st, s);
}

// (One cluster sorts whatever the batch: 262144 places into 32768 x 256 take 214 us, 1048576 into 50000 x 64 773.)
// Eight CTAs sort faster (32768 places 23 us, four 34) but leave fewer to fill (65536 x 2048: 92 us and 80): they are taken where the sort,
// about 1 ns a place by four, would take longer than the zeros, 0.8 ps an element.
cudaError_t sort_places(const SortArgs& s, bool wide, cudaStream_t st) {
    if (s.tokens <= kSmallTokens) return wide ? launch_sort<int64_t, 1>(s, st) : launch_sort<int32_t, 1>(s, st);
    if (s.tokens * 1024 > s.vocab * s.width) return wide ? launch_sort<int64_t, 8>(s, st) : launch_sort<int32_t, 8>(s, st);
    return wide ? launch_sort<int64_t, 4>(s, st) : launch_sort<int32_t, 4>(s, st);
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
    return (size_t)(2 * up256(tokens * 8) + up256((1 + chunks) * 4) + up256(chunks * 2 * width * 4));
}

tng_status tng_embed_grad(const void* dy_dev, tng_dtype type, uint64_t tokens, uint64_t width, uint64_t lddy, const void* ids_dev,
                          uint32_t id_bytes, uint64_t vocab, float scale, float* dtable_dev, uint64_t ldd, void* scratch_dev, void* stream) {
    if (!type_ok(type) || width < 1 || width >= (1u << 25) || vocab < 1 || !dims_ok(tokens, width) || !dims_ok(vocab, width) || (id_bytes != 4 && id_bytes != 8) ||
        !matrix_ok(dtable_dev, TNG_F32, width, ldd))
        return TNG_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (tokens == 0) return layer_status(cudaMemset2DAsync(dtable_dev, ldd * 4, 0, width * 4, vocab, st));
    if (!matrix_ok(dy_dev, type, width, lddy) || !ids_dev || !aligned(ids_dev, id_bytes) || !scratch_dev || !aligned(scratch_dev, 256)) return TNG_ERR_INVALID_ARG;
    unsigned char* at = static_cast<unsigned char*>(scratch_dev);
    SortArgs s = {};
    s.ids = ids_dev; s.tokens = tokens; s.vocab = vocab; s.ldd = ldd; s.dtable = dtable_dev; s.width = (uint32_t)width;
    const uint64_t list = up256(tokens * 8);
    for (int i = 0; i < 2; ++i) s.pair[i] = reinterpret_cast<uint2*>(at + i * list);
    const uint64_t chunk = chunk_of(tokens), chunks = (tokens + chunk - 1) / chunk, spans = (width + kGradSpan - 1) / kGradSpan;
    uint32_t* crossing = reinterpret_cast<uint32_t*>(at + 2 * list);
    float* parts = reinterpret_cast<float*>(at + 2 * list + up256((1 + chunks) * 4));
    s.crossing = crossing;
    uint32_t bits = 1;
    while (vocab >> bits) ++bits;                          // of the largest key, vocab itself
    s.passes = (bits + 8) / 9;
    s.bits = (bits + s.passes - 1) / s.passes;
    const bool wide = id_bytes == 8;
    cudaError_t e = sort_places(s, wide, st);
    if (e != cudaSuccess) return layer_status(e);
    const GradArgs g{dy_dev, s.pair[0], crossing, crossing + 1, parts, dtable_dev, tokens, vocab, lddy, ldd,
                     (uint32_t)width, (uint32_t)chunk, (uint32_t)chunks, scale};
    const dim3 grid((unsigned)chunks, (unsigned)spans);
    e = with_type(type, [&](auto t) {
        using T = decltype(t);
        const bool vec = aligned(dy_dev, 16) && (tokens == 1 || lddy * sizeof(T) % 16 == 0);
        return launch_layer(vec ? embed_sum_kernel<T, true> : embed_sum_kernel<T, false>, grid, kGradThreads, 0, 1, st, g);
    });
    if (e == cudaSuccess && chunks > 1) {
        const uint64_t most = (chunks - 1) * ((width + kJoinSpan - 1) / kJoinSpan), cap = 8ull * sm_count_now();
        e = launch_layer(embed_join_kernel, (unsigned)(most < cap ? most : cap), kJoinThreads, 0, 1, st, g);
    }
    return layer_status(e);
}

}  // extern "C"
