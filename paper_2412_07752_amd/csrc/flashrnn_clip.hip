// Clipping of many gradient tensors by their global norm (include/flashrnn.h).
#include "flashrnn_rows.h"

using namespace flashrnn;

namespace {

constexpr int kTensors = 128;      // tensors per launch: their table is a kernel argument, which holds 4 KB
constexpr int kMaxBlocks = 2048;   // workgroups per launch, each with a partial sum
constexpr int kChunk = 8192;       // values of one tensor that a workgroup takes at a time

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

template <typename F> __device__ __forceinline__ void for_chunks(const Table& t, F&& f) {
    for (int chunk = blockIdx.x; chunk < t.first_chunk[t.count]; chunk += gridDim.x) {
        const int k = tensor_of(t, chunk);
        const size_t n = (size_t)(t.size[k] < 0 ? ~t.size[k] : t.size[k]), begin = (size_t)(chunk - t.first_chunk[k]) * kChunk;
        const size_t end = begin + kChunk < n ? begin + kChunk : n;
        if (t.size[k] < 0) f((const __bf16*)t.in[k], (__bf16*)t.out[k], begin, end);
        else f((const float*)t.in[k], (float*)t.out[k], begin, end);
    }
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(Table t, double* __restrict__ part) {
    __shared__ double lds[kThreads / kWave];
    double s = 0.0;
    for_chunks(t, [&](auto* in, auto*, size_t begin, size_t end) {
        for (size_t j = begin + threadIdx.x; j < end; j += kThreads) {
            const double v = load_value(in + j);
            s += v * v;
        }
    });
    s = block_sum<kThreads>(s, lds);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// the norm, and the factor behind the partial sums
__global__ __launch_bounds__(kThreads) void grad_factor_kernel(double* __restrict__ part, int count, float max_norm, float* __restrict__ norm_out) {
    __shared__ double lds[kThreads / kWave];
    double s = 0.0;
    for (int i = threadIdx.x; i < count; i += kThreads) s += part[i];
    const double norm = sqrt(block_sum<kThreads>(s, lds));
    if (threadIdx.x == 0) {
        norm_out[0] = (float)norm;
        part[count] = norm <= max_norm ? 1.0 : max_norm / norm;
    }
}

__global__ __launch_bounds__(kThreads) void grad_scale_kernel(Table t, const double* __restrict__ factor_in) {
    const float factor = (float)*factor_in;
    for_chunks(t, [&](auto* in, auto* out, size_t begin, size_t end) {
        if (in == out && factor == 1.f) return;
        for (size_t j = begin + threadIdx.x; j < end; j += kThreads) store_value(out + j, load_value(in + j) * factor);
    });
}

int tables_of(int count) { return count / kTensors + (count % kTensors != 0); }

}  // namespace

extern "C" {

size_t flashrnn_grad_clip_workspace_bytes(int count) {
    if (count < 0) return 0;
    return ((size_t)tables_of(count) * kMaxBlocks + 1) * sizeof(double) / 256 * 256 + 256;
}

int flashrnn_grad_clip(int count, const void* const* grads, void* const* out, const long long* sizes, const int* dtypes, float max_norm, void* norm, void* workspace,
                       void* hip_stream) {
    if (count < 0 || !(max_norm >= 0.f)) return FLASHRNN_ERR_SHAPE;
    if (!norm || (count && (!grads || !sizes || !dtypes))) return FLASHRNN_ERR_NULL;
    if (!workspace || !aligned_to(workspace, 256)) return FLASHRNN_ERR_WORKSPACE;
    if (!aligned_to(norm, 4)) return FLASHRNN_ERR_UNSUPPORTED;
    for (int k = 0; k < count; ++k) {
        if (sizes[k] < 0 || !is_io_type(dtypes[k])) return FLASHRNN_ERR_SHAPE;
        if (sizes[k] && (!grads[k] || (out && !out[k]))) return FLASHRNN_ERR_NULL;
        if (!aligned_to(grads[k], type_size(dtypes[k])) || (out && !aligned_to(out[k], type_size(dtypes[k])))) return FLASHRNN_ERR_UNSUPPORTED;
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
    hipLaunchKernelGGL(grad_factor_kernel, dim3(1), dim3(kThreads), 0, stream, part, parts, max_norm, (float*)norm);
    if (const int e = launch_status()) return e;
    if (!out) return FLASHRNN_OK;
    for (int first = 0; first < count; first += kTensors) {
        const int blocks = fill(first);
        if (blocks == 0) continue;
        hipLaunchKernelGGL(grad_scale_kernel, dim3(blocks), dim3(kThreads), 0, stream, t, (const double*)(part + parts));
        if (const int e = launch_status()) return e;
    }
    return FLASHRNN_OK;
}

}  // extern "C"
