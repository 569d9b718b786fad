// Embedding lookup and its gradient by sorted tokens (include/flashrnn.h).
//
// The gradient sorts the places by their word (stable, so that the places of a word stay in order) with a radix sort of digits of up to
// kDigitBits bits, least significant first.  Per digit: every workgroup counts the digits of its kTile places, then every workgroup adds up
// the counts of smaller digits and of the workgroups before it and moves its places behind them.  Tokens outside the vocabulary
// sort behind all words.
#include "flashrnn_rows.h"

using namespace flashrnn;

namespace {

constexpr int kWaves = kThreads / kWave;
constexpr int kDigitBits = 8;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kTile = 2048;   // places per workgroup of the sort

template <typename I> __device__ __forceinline__ uint32_t key_of(const I* tokens, size_t i, uint32_t vocab) {
    const int64_t t = tokens[i];
    return t >= 0 && t < (int64_t)vocab ? (uint32_t)t : vocab;
}

template <typename E, typename O, typename I>
__global__ __launch_bounds__(kThreads) void embedding_fwd_kernel(size_t n, int vocab, int width, const E* __restrict__ table, const I* __restrict__ tokens, O* __restrict__ out, float scale) {
    for (size_t row = blockIdx.x; row < n; row += gridDim.x) {
        const int64_t t = tokens[row];
        const bool there = t >= 0 && t < vocab;
        for (int j = threadIdx.x; j < width; j += kThreads) store_value(out + row * width + j, there ? load_value(table + (size_t)t * width + j) * scale : 0.f);
    }
}

// counts[digit][workgroup]; keys == nullptr: the first digit, straight from the tokens
template <typename I>
__global__ __launch_bounds__(kThreads) void count_digits_kernel(const I* __restrict__ tokens, const uint32_t* __restrict__ keys, size_t n, uint32_t vocab, int shift,
                                                                uint32_t* __restrict__ counts) {
    __shared__ uint32_t lds[kDigits];
    for (int d = threadIdx.x; d < kDigits; d += kThreads) lds[d] = 0;
    __syncthreads();
    for (int u = threadIdx.x; u < kTile; u += kThreads) {
        const size_t i = (size_t)blockIdx.x * kTile + u;
        if (i < n) atomicAdd(&lds[(keys ? keys[i] : key_of(tokens, i, vocab)) >> shift & (kDigits - 1)], 1u);   // (whole numbers: any order)
    }
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kThreads) counts[(size_t)d * gridDim.x + blockIdx.x] = lds[d];
}

// exclusive sums over counts[digit][workgroup], by one workgroup
__global__ __launch_bounds__(1024) void scan_counts_kernel(uint32_t* __restrict__ counts, size_t n) {
    __shared__ uint32_t lds[1024];
    uint32_t before = 0;
    for (size_t at = 0; at < n; at += 1024) {
        const size_t i = at + threadIdx.x;
        const uint32_t v = i < n ? counts[i] : 0;
        lds[threadIdx.x] = v;
        __syncthreads();
        for (int o = 1; o < 1024; o <<= 1) {
            const uint32_t a = threadIdx.x >= (unsigned)o ? lds[threadIdx.x - o] : 0;
            __syncthreads();
            lds[threadIdx.x] += a;
            __syncthreads();
        }
        if (i < n) counts[i] = before + lds[threadIdx.x] - v;
        before += lds[1023];
        __syncthreads();
    }
}

// A wave takes the 64 places of a run in order: lanes with the same digit find each other by comparing the digits' bits, and the lane's place
// among them is the number of lower lanes.  Waves take runs of their own behind one another: wave w the runs w * kRuns, ...
template <typename I>
__global__ __launch_bounds__(kThreads) void move_places_kernel(const I* __restrict__ tokens, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ places, size_t n,
                                                               uint32_t vocab, int shift, const uint32_t* __restrict__ offsets, uint32_t* __restrict__ keys_out,
                                                               uint32_t* __restrict__ places_out) {
    constexpr int kRuns = kTile / kThreads;
    __shared__ uint32_t lds[kWaves][kDigits];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int d = threadIdx.x; d < kWaves * kDigits; d += kThreads) lds[0][d] = 0;
    __syncthreads();
    uint32_t key[kRuns], rank[kRuns];
#pragma unroll
    for (int u = 0; u < kRuns; ++u) {
        const size_t i = (size_t)blockIdx.x * kTile + (w * kRuns + u) * kWave + lane;
        const bool in = i < n;
        key[u] = in ? (keys ? keys[i] : key_of(tokens, i, vocab)) : 0;
        const uint32_t d = key[u] >> shift & (kDigits - 1);
        uint64_t same = __ballot(in);
#pragma unroll
        for (int b = 0; b < kDigitBits; ++b) {
            const uint64_t m = __ballot(d >> b & 1);
            same &= d >> b & 1 ? m : ~m;
        }
        const uint32_t lower = __popcll(same & ((1ull << lane) - 1));
        const uint32_t base = lds[w][d];   // (one wave, one row: its LDS accesses are in order)
        rank[u] = base + lower;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (in && lower == 0) lds[w][d] = base + __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kThreads) {
        uint32_t at = offsets[(size_t)d * gridDim.x + blockIdx.x];
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
            const uint32_t c = lds[v][d];
            lds[v][d] = at;
            at += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kRuns; ++u) {
        const size_t i = (size_t)blockIdx.x * kTile + (w * kRuns + u) * kWave + lane;
        if (i >= n) continue;
        const uint32_t to = lds[w][key[u] >> shift & (kDigits - 1)] + rank[u];
        keys_out[to] = key[u];
        places_out[to] = places ? places[i] : (uint32_t)i;
    }
}

// the first sorted place whose word is v or a later one
__device__ __forceinline__ size_t first_of(const uint32_t* keys, size_t n, uint32_t v) {
    size_t lo = 0, hi = n;
    while (lo < hi) {
        const size_t mid = (lo + hi) / 2;
        if (keys[mid] < v) lo = mid + 1; else hi = mid;
    }
    return lo;
}

template <typename O>
__global__ __launch_bounds__(kThreads) void sum_places_kernel(const uint32_t* __restrict__ keys, const uint32_t* __restrict__ places, size_t n, int vocab, int width, const O* __restrict__ dout,
                                                              float* __restrict__ dtable, float scale, int accumulate) {
    for (uint32_t v = blockIdx.x; v < (uint32_t)vocab; v += gridDim.x) {
        const size_t begin = first_of(keys, n, v), end = first_of(keys, n, v + 1);
        if (begin == end && accumulate) continue;
        for (int j = threadIdx.x; j < width; j += kThreads) {
            float s = 0.f;
            for (size_t p = begin; p < end; ++p) s += load_value(dout + (size_t)places[p] * width + j);
            s *= scale;
            float* out = dtable + (size_t)v * width + j;
            *out = accumulate ? *out + s : s;
        }
    }
}

int check_desc(const flashrnn_embedding_desc_t* d) {
    if (!d) return FLASHRNN_ERR_NULL;
    if (d->tokens < 0 || d->vocab <= 0 || d->width <= 0) return FLASHRNN_ERR_SHAPE;
    if (!is_io_type(d->table_dtype) || !is_io_type(d->io_dtype) || !is_index_type(d->index_dtype)) return FLASHRNN_ERR_SHAPE;
    if (d->tokens > 2147483647LL) return FLASHRNN_ERR_UNSUPPORTED;
    return FLASHRNN_OK;
}

struct Workspace {
    size_t tiles, keys[2], places[2], counts, total;
};
Workspace workspace_of(const flashrnn_embedding_desc_t* d) {
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    Workspace w;
    const size_t list = up((size_t)d->tokens * 4);
    w.tiles = ((size_t)d->tokens + kTile - 1) / kTile;
    size_t at = 0;
    for (int i = 0; i < 2; ++i) {
        w.keys[i] = at; at += list;
        w.places[i] = at; at += list;
    }
    w.counts = at;
    w.total = at + up(w.tiles * kDigits * 4) + 256;
    return w;
}

}  // namespace

extern "C" {

size_t flashrnn_embedding_workspace_bytes(const flashrnn_embedding_desc_t* d) { return check_desc(d) == FLASHRNN_OK ? workspace_of(d).total : 0; }

int flashrnn_embedding_fwd(const flashrnn_embedding_desc_t* d, const void* table, const void* tokens, void* out, void* hip_stream) {
    const int rc = check_desc(d);
    if (rc != FLASHRNN_OK) return rc;
    if (d->tokens == 0) return FLASHRNN_OK;
    if (!table || !tokens || !out) return FLASHRNN_ERR_NULL;
    if (!aligned_to(table, type_size(d->table_dtype)) || !aligned_to(out, type_size(d->io_dtype)) || !aligned_to(tokens, type_size(d->index_dtype))) return FLASHRNN_ERR_UNSUPPORTED;
    return with_io_type(d->table_dtype, [&](auto* et) {
        return with_io_type(d->io_dtype, [&](auto* ot) {
            return with_index_type(d->index_dtype, [&](auto* it) {
                using E = std::remove_pointer_t<decltype(et)>;
                using O = std::remove_pointer_t<decltype(ot)>;
                using I = std::remove_pointer_t<decltype(it)>;
                hipLaunchKernelGGL((embedding_fwd_kernel<E, O, I>), dim3(row_blocks((size_t)d->tokens)), dim3(kThreads), 0, (hipStream_t)hip_stream, (size_t)d->tokens, d->vocab, d->width, (const E*)table,
                                   (const I*)tokens, (O*)out, d->scale);
                return launch_status();
            });
        });
    });
}

int flashrnn_embedding_bwd(const flashrnn_embedding_desc_t* d, const void* tokens, const void* dout, void* dtable, int accumulate, void* workspace, void* hip_stream) {
    const int rc = check_desc(d);
    if (rc != FLASHRNN_OK) return rc;
    const size_t n = (size_t)d->tokens;
    if (!dtable || (n && (!tokens || !dout))) return FLASHRNN_ERR_NULL;
    if (!workspace || !aligned_to(workspace, 256)) return FLASHRNN_ERR_WORKSPACE;
    if (!aligned_to(dout, type_size(d->io_dtype)) || !aligned_to(tokens, type_size(d->index_dtype)) || !aligned_to(dtable, 4)) return FLASHRNN_ERR_UNSUPPORTED;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const Workspace w = workspace_of(d);
    char* ws = (char*)workspace;
    uint32_t *keys = nullptr, *places = nullptr, *counts = (uint32_t*)(ws + w.counts);
    const unsigned tiles = (unsigned)w.tiles;
    if (n) {
        int bits = 0;
        while (bits < 32 && (uint64_t)d->vocab >> bits) ++bits;   // keys go up to vocab itself
        for (int shift = 0, pass = 0; shift < bits; shift += kDigitBits, ++pass) {
            uint32_t *keys_to = (uint32_t*)(ws + w.keys[pass & 1]), *places_to = (uint32_t*)(ws + w.places[pass & 1]);
            const int e = with_index_type(d->index_dtype, [&](auto* it) {
                using I = std::remove_pointer_t<decltype(it)>;
                hipLaunchKernelGGL((count_digits_kernel<I>), dim3(tiles), dim3(kThreads), 0, stream, (const I*)tokens, (const uint32_t*)keys, n, (uint32_t)d->vocab, shift, counts);
                if (const int err = launch_status()) return err;
                hipLaunchKernelGGL(scan_counts_kernel, dim3(1), dim3(1024), 0, stream, counts, (size_t)tiles * kDigits);
                if (const int err = launch_status()) return err;
                hipLaunchKernelGGL((move_places_kernel<I>), dim3(tiles), dim3(kThreads), 0, stream, (const I*)tokens, (const uint32_t*)keys, (const uint32_t*)places, n,
                                   (uint32_t)d->vocab, shift, (const uint32_t*)counts, keys_to, places_to);
                return launch_status();
            });
            if (e != FLASHRNN_OK) return e;
            keys = keys_to;
            places = places_to;
        }
    }
    return with_io_type(d->io_dtype, [&](auto* ot) {
        using O = std::remove_pointer_t<decltype(ot)>;
        hipLaunchKernelGGL((sum_places_kernel<O>), dim3(row_blocks((size_t)d->vocab)), dim3(kThreads), 0, stream, (const uint32_t*)keys, (const uint32_t*)places, n, d->vocab, d->width, (const O*)dout,
                           (float*)dtable, d->scale, accumulate);
        return launch_status();
    });
}

}  // extern "C"
