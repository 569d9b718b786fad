// Shared by the kernels around the time-step loop (embedding, layer norm, cross entropy, clipping): element types and sums over lanes.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "flashrnn.h"
#include "flashrnn_common.h"

namespace flashrnn {

constexpr int kWave = 64;

inline bool is_io_type(int t) { return t == FLASHRNN_F32 || t == FLASHRNN_BF16; }
inline bool is_index_type(int t) { return t == FLASHRNN_I32 || t == FLASHRNN_I64; }
inline size_t type_size(int t) { return t == FLASHRNN_BF16 ? 2 : t == FLASHRNN_I64 ? 8 : 4; }
inline bool aligned_to(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline int launch_status() { return hipGetLastError() == hipSuccess ? FLASHRNN_OK : FLASHRNN_ERR_LAUNCH; }

// workgroups of a kernel that takes rows blockIdx.x, blockIdx.x + gridDim.x, ... (a dispatch holds fewer than 2^32 threads)
inline unsigned row_blocks(size_t rows) { return (unsigned)(rows < (1u << 20) ? rows : (1u << 20)); }

// one value of a tensor of either type
__device__ __forceinline__ float load_value(const float* p) { return *p; }
__device__ __forceinline__ float load_value(const __bf16* p) { return (float)*p; }
__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_value(__bf16* p, float v) { *p = (__bf16)v; }

// sum over the threads of a workgroup of NT threads, the same in every thread; `lds` holds NT / 64 values
template <int NT, typename T> __device__ __forceinline__ T block_sum(T v, T* lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();   // (the values of an earlier call have been read)
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    T s = 0;
#pragma unroll
    for (int i = 0; i < NT / kWave; ++i) s += lds[i];
    return s;
}
template <int NT> __device__ __forceinline__ float block_max(float v, float* lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = lds[0];
#pragma unroll
    for (int i = 1; i < NT / kWave; ++i) s = fmaxf(s, lds[i]);
    return s;
}

// calls f with a null pointer of the C++ type behind a flashrnn_dtype_t / flashrnn_index_t
template <typename F> int with_io_type(int t, F&& f) { return t == FLASHRNN_BF16 ? f((__bf16*)nullptr) : f((float*)nullptr); }
template <typename F> int with_index_type(int t, F&& f) { return t == FLASHRNN_I64 ? f((int64_t*)nullptr) : f((int32_t*)nullptr); }

}  // namespace flashrnn
