// Clipping of many gradient tensors by their global norm (include/flashrnn.h).
//
// norm = sqrt(sum g^2), out = g min(1, max_norm / norm).  Bound by memory: two reads, the second behind the norm, and a write.  Tensors of any number and size are cut into chunks that workgroups take in a
// fixed order; the tensors' places travel as a kernel argument, so that a call keeps nothing and can be captured.  330 M float32 values out of place 707 us: norm 214 us (6.2 TB/s), products 491 us
// (5.4 TB/s).  A single layer's 49,000 values: 3.6 and 4.7 us, one launch behind the other.  (All values by one workgroup, in one launch: 5.6 us for 2000 of them, where the two launches, bound by the host,
// take 7.5 to 9.8; but 9.6 for 49,500 and 19 for 21 tensors.)
#include "flashrnn_rows.h"

using namespace flashrnn;

namespace {

constexpr int kTensors = 128;      // tensors per launch: their table is a kernel argument, which holds 4 KB (with 16 a small call takes as long)
constexpr int kMaxBlocks = 1024;   // workgroups per launch, each with a partial sum (683 MB of bf16 values 330 us, with 2048 workgroups 364; 1.3 GB of float32 714 and 726)
constexpr int kMaxCount = 1 << 24;
constexpr int kChunk = 8192;       // values of one tensor that a workgroup takes at a time (32 KB whatever the type, the tensor found by a ballot, the first loads ahead of the norm: 4.4 + 5.7 us a small call, 1.3 GB 755)

struct Table {
    const void* in[kTensors];
    void* out[kTensors];
    long long size[kTensors];        // values; ~values where they are bf16
    int first_chunk[kTensors + 1];   // chunks of the tensors before
    int count;
};
static_assert(sizeof(Table) <= 3840, "kernel arguments");

__device__ __forceinline__ int tensor_of(const Table& t, int chunk) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {   // the last tensor that starts at or before the chunk (an empty one starts where the next one does)
        const int mid = (lo + hi + 1) >> 1;
        if (t.first_chunk[mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// f(in, out, values) for chunks blockIdx.x, blockIdx.x + gridDim.x, ...; BACK: from the last one back.  The second kernel begins with what the first one read last and the last-level cache may
// still hold (its own output goes past the caches): 683 MB of bf16 values 338 us and 359, 292 MB of float32 148 and 153, 1.3 GB 709 and 717.
template <bool BACK, typename F> __device__ __forceinline__ void for_chunks(const Table& t, F&& f) {
    const int chunks = t.first_chunk[t.count];
    for (int i = blockIdx.x; i < chunks; i += gridDim.x) {
        const int chunk = BACK ? chunks - 1 - i : i;
        const int k = tensor_of(t, chunk);
        const long long n = t.size[k] < 0 ? ~t.size[k] : t.size[k], begin = (long long)(chunk - t.first_chunk[k]) * kChunk;
        const int count = n - begin < kChunk ? (int)(n - begin) : kChunk;
        if (t.size[k] < 0) f((const __bf16*)t.in[k] + begin, (__bf16*)t.out[k] + begin, count);
        else f((const float*)t.in[k] + begin, (float*)t.out[k] + begin, count);
    }
}

// The sum of the squares, in 64 bits: a float32 square may leave float32's range, and its sum over a model's gradients loses the small tensors.
__global__ __launch_bounds__(kThreads) void grad_norm_kernel(Table t, double* __restrict__ part) {
    __shared__ double lds[kThreads / kWave];
    double s = 0.0;
    auto add = [&](float x) {
        const double v = x;
        s = fma(v, v, s);
    };
    for_chunks<false>(t, [&](auto* in, auto*, int count) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(in)>>;
        constexpr int V = 16 / sizeof(T), kRounds = kChunk / (kThreads * V);
        if (count == kChunk) {
            Chunk<T, V> c[kRounds];
#pragma unroll
            for (int u = 0; u < kRounds; ++u) c[u].load(in + (u * kThreads + threadIdx.x) * V);
#pragma unroll
            for (int u = 0; u < kRounds; ++u)
#pragma unroll
                for (int i = 0; i < V; ++i) add(c[u].get(i));
        } else {
            for (int at = threadIdx.x * V; at < count; at += kThreads * V) {
                if (at + V <= count) {
                    Chunk<T, V> c;
                    c.load(in + at);
#pragma unroll
                    for (int i = 0; i < V; ++i) add(c.get(i));
                } else {
                    for (int i = at; i < count; ++i) add(load_value(in + i));
                }
            }
        }
    });
    s = block_sum<kThreads>(s, lds);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The norm and the factor from all partial sums, in every workgroup the same (a launch of its own for them takes longer than reading them again), then the products.
__global__ __launch_bounds__(kThreads) void grad_scale_kernel(Table t, const double* __restrict__ part, int parts, float max_norm, float* __restrict__ norm_out, bool stream) {
    __shared__ double lds[kThreads / kWave];
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) s += part[i];
    const double norm = sqrt(block_sum<kThreads>(s, lds));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const double exact = norm <= max_norm ? 1.0 : max_norm / norm;
    const float factor = (float)exact;
    // times: a value's product with the factor
    auto scale = [&](auto times) __attribute__((always_inline)) {
        for_chunks<true>(t, [&](auto* in, auto* out, int count) {
            using T = std::remove_pointer_t<decltype(out)>;
            constexpr int V = 16 / sizeof(T), kRounds = kChunk / (kThreads * V);
            if (in == out && factor == 1.f) return;
            auto put = [&](const Chunk<T, V>& c, int at) {
                float v[V];
                Chunk<T, V> o;
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = times(c.get(i));
                o.put(v);
                o.store(out + at, stream);
            };
            if (count == kChunk) {
                Chunk<T, V> c[kRounds];
#pragma unroll
                for (int u = 0; u < kRounds; ++u) c[u].load(in + (u * kThreads + threadIdx.x) * V);
#pragma unroll
                for (int u = 0; u < kRounds; ++u) put(c[u], (u * kThreads + threadIdx.x) * V);
            } else {
                for (int at = threadIdx.x * V; at < count; at += kThreads * V) {
                    if (at + V <= count) {
                        Chunk<T, V> c;
                        c.load(in + at);
                        put(c, at);
                    } else {
                        for (int i = at; i < count; ++i) store_value(out + i, times(load_value(in + i)));
                    }
                }
            }
        });
    };
    // Below float32's smallest normal number the factor would lose its digits, while its products with gradients of the norm's size do not: there it is 0.5 to 1 times 2^power, and the product takes the power
    // (a loop of its own: the instruction for it in every product made 683 MB of bf16 values 343 us instead of 338).
    if (exact > 0.0 && exact < (double)__FLT_MIN__) {
        const float part = (float)__builtin_amdgcn_frexp_mant(exact);
        const int power = __builtin_amdgcn_frexp_exp(exact);
        scale([&](float v) __attribute__((always_inline)) { return __builtin_amdgcn_ldexpf(v * part, power); });
    } else {
        scale([&](float v) __attribute__((always_inline)) { return v * factor; });
    }
}

int tables_of(int count) { return count / kTensors + (count % kTensors != 0); }

}  // namespace

extern "C" {

size_t flashrnn_grad_clip_workspace_bytes(int count) {
    if (count < 0 || count > kMaxCount) return 0;
    return ((size_t)tables_of(count) * kMaxBlocks + 1) * sizeof(double) / 256 * 256 + 256;
}

int flashrnn_grad_clip(int count, const void* const* grads, void* const* out, const long long* sizes, const int* dtypes, float max_norm, void* norm, void* workspace,
                       void* hip_stream) {
    if (count < 0 || !(max_norm >= 0.f)) return FLASHRNN_ERR_SHAPE;
    if (count > kMaxCount) return FLASHRNN_ERR_UNSUPPORTED;
    if (!norm || (count && (!grads || !sizes || !dtypes))) return FLASHRNN_ERR_NULL;
    if (!workspace || !aligned_to(workspace, 256)) return FLASHRNN_ERR_WORKSPACE;
    if (!aligned_to(norm, 4)) return FLASHRNN_ERR_UNSUPPORTED;
    double bytes = 0;
    for (int k = 0; k < count; ++k) {
        if (sizes[k] < 0 || !is_io_type(dtypes[k])) return FLASHRNN_ERR_SHAPE;
        if (sizes[k] && (!grads[k] || (out && !out[k]))) return FLASHRNN_ERR_NULL;
        if (!aligned_to(grads[k], type_size(dtypes[k])) || (out && !aligned_to(out[k], type_size(dtypes[k])))) return FLASHRNN_ERR_UNSUPPORTED;
        bytes += (double)sizes[k] * type_size(dtypes[k]);
        if (sizes[k] > (1LL << 40)) return FLASHRNN_ERR_UNSUPPORTED;   // (chunks of a table are counted in 32 bits)
    }
    const hipStream_t stream = (hipStream_t)hip_stream;
    double* part = (double*)workspace;
    int parts = 0;
    Table t;
    auto fill = [&](int first) {   // the table of tensors first, first + 1, ...; its workgroups
        long long chunks = 0;
        t.count = 0;
        for (int k = first; k < count && t.count < kTensors; ++k) {
            t.in[t.count] = grads[k];
            t.out[t.count] = out ? out[k] : nullptr;
            t.size[t.count] = dtypes[k] == FLASHRNN_BF16 ? ~sizes[k] : sizes[k];
            t.first_chunk[t.count++] = (int)chunks;
            chunks += (sizes[k] + kChunk - 1) / kChunk;
            if (chunks > 0x40000000LL) return -1;
        }
        t.first_chunk[t.count] = (int)chunks;
        return chunks < kMaxBlocks ? (int)chunks : kMaxBlocks;
    };
    for (int first = 0; first < count; first += kTensors)
        if (fill(first) < 0) return FLASHRNN_ERR_UNSUPPORTED;
    for (int first = 0; first < count; first += kTensors) {
        const int blocks = fill(first);
        if (blocks == 0) continue;
        hipLaunchKernelGGL(grad_norm_kernel, dim3(blocks), dim3(kThreads), 0, stream, t, part + parts);
        if (const int e = launch_status()) return e;
        parts += blocks;
    }
    // (a table without values, or no table: a launch that leaves the norm alone)
    bool told = false;
    for (int first = 0; first < count || !told; first += kTensors) {
        const int blocks = out ? fill(first) : 0;
        if (blocks == 0) {
            if (told || first + kTensors < count) continue;
            t.count = 0;
            t.first_chunk[0] = 0;
        }
        hipLaunchKernelGGL(grad_scale_kernel, dim3(blocks ? blocks : 1), dim3(kThreads), 0, stream, t, (const double*)part, parts, max_norm, told ? nullptr : (float*)norm,
                           bytes > kStreamBytes);
        if (const int e = launch_status()) return e;
        told = true;
    }
    return FLASHRNN_OK;
}

}  // extern "C"
