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

// Outputs larger than the second-level caches (eight of 4 MB) are stored past them: layer norm of 65536 x 8 x 256 states 140 us and 148, of 65536 x 2048 values in bf16 90 us and 92.
constexpr size_t kStreamBytes = 32u << 20;

// one value of a tensor of either type
__device__ __forceinline__ float load_value(const float* p) { return *p; }
__device__ __forceinline__ float load_value(const __bf16* p) { return (float)*p; }
__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_value(__bf16* p, float v) { *p = (__bf16)v; }

// V consecutive values of a tensor as they lie in memory, moved in words of up to 16 bytes from any place that the element's own size divides
// (global memory takes wide accesses at such addresses: a row of odd length costs no scalar loads).
typedef int i32x4_any __attribute__((vector_size(16), aligned(2)));
typedef int i32x2_any __attribute__((vector_size(8), aligned(2)));

template <typename T, int V> struct Chunk {
    static constexpr int W = V * (int)sizeof(T) / 4;   // 32-bit words
    static_assert(W == 2 || W % 4 == 0, "whole wide accesses");
    uint32_t w[W];

    __device__ __forceinline__ void load(const T* p) {
        if constexpr (W == 2) {
            const i32x2_any a = *(const i32x2_any*)p;
            w[0] = a[0];
            w[1] = a[1];
        } else {
#pragma unroll
            for (int i = 0; i < W / 4; ++i) {
                const i32x4_any a = ((const i32x4_any*)p)[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[4 * i + j] = a[j];
            }
        }
    }
    // stream: past the caches, for outputs that these cannot hold
    __device__ __forceinline__ void store(T* p, bool stream = false) const {
        if constexpr (W == 2) {
            const i32x2_any a = {(int)w[0], (int)w[1]};
            if (stream) __builtin_nontemporal_store(a, (i32x2_any*)p);
            else *(i32x2_any*)p = a;
        } else {
#pragma unroll
            for (int i = 0; i < W / 4; ++i) {
                const i32x4_any a = {(int)w[4 * i], (int)w[4 * i + 1], (int)w[4 * i + 2], (int)w[4 * i + 3]};
                if (stream) __builtin_nontemporal_store(a, (i32x4_any*)p + i);
                else ((i32x4_any*)p)[i] = a;
            }
        }
    }
    __device__ __forceinline__ float get(int i) const {   // (i: known when compiled)
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[i]);
        else return __builtin_bit_cast(float, i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
    __device__ __forceinline__ void put(const float (&v)[V]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < V; ++i) w[i] = __builtin_bit_cast(uint32_t, v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        }
    }
};
template <int V> __device__ __forceinline__ void load_chunk(const void* base, bool bf16, size_t at, float (&v)[V]) {   // (of a type that is not known when compiled)
    if (bf16) {
        Chunk<__bf16, V> c;
        c.load((const __bf16*)base + at);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = c.get(i);
    } else {
        Chunk<float, V> c;
        c.load((const float*)base + at);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = c.get(i);
    }
}
template <int V> __device__ __forceinline__ void store_chunk(void* base, bool bf16, size_t at, const float (&v)[V], bool stream) {
    if (bf16) {
        Chunk<__bf16, V> c;
        c.put(v);
        c.store((__bf16*)base + at, stream);
    } else {
        Chunk<float, V> c;
        c.put(v);
        c.store((float*)base + at, stream);
    }
}

// sum over groups of L lanes, the same in every lane (all lanes of the wave take part)
template <int L> __device__ __forceinline__ float lanes_sum(float v) {
    static_assert(L == 8 || L == 16 || L == 32 || L == 64, "lanes of a wave");
#define FLASHRNN_DPP(x, ctrl) __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, 0xF, 0xF, false))
    v += FLASHRNN_DPP(v, 0xB1);    // lane ^ 1
    v += FLASHRNN_DPP(v, 0x4E);    // lane ^ 2
    v += FLASHRNN_DPP(v, 0x141);   // 7 - lane: the other four of eight
    if constexpr (L >= 16) v += FLASHRNN_DPP(v, 0x140);   // 15 - lane
#undef FLASHRNN_DPP
    if constexpr (L >= 32) {   // rows of 16 lanes, then halves of 32, exchanged between two copies
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        const auto p = __builtin_amdgcn_permlane16_swap(b, b, false, false);
        const uint32_t x = p[0], y = p[1];
        v = __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
    }
    if constexpr (L >= 64) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        const auto p = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        const uint32_t x = p[0], y = p[1];
        v = __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
    }
    return v;
}
// sum over a group of L threads: lanes of a wave, or a whole workgroup of L threads, whose waves meet in slot (two slots taken in turn need no other barrier)
template <int L> __device__ __forceinline__ float group_sum(float v, float* slot) {
    if constexpr (L <= kWave) {
        return lanes_sum<L>(v);
    } else {
        v = lanes_sum<kWave>(v);
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
        __syncthreads();
        float s = slot[0];
#pragma unroll
        for (int i = 1; i < L / kWave; ++i) s += slot[i];
        return s;
    }
}

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
