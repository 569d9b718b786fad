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
    // stream: past the caches, for outputs that these cannot hold.  (The empty asm keeps the compiler from joining the two stores into one that is neither.)
    __device__ __forceinline__ void store(T* p, bool stream = false) const {
        if constexpr (W == 2) {
            const i32x2_any a = {(int)w[0], (int)w[1]};
            if (stream) {
                asm volatile("");
                __builtin_nontemporal_store(a, (i32x2_any*)p);
                asm volatile("");
            } else {
                *(i32x2_any*)p = a;
            }
        } else {
#pragma unroll
            for (int i = 0; i < W / 4; ++i) {
                const i32x4_any a = {(int)w[4 * i], (int)w[4 * i + 1], (int)w[4 * i + 2], (int)w[4 * i + 3]};
                if (stream) {
                    asm volatile("");
                    __builtin_nontemporal_store(a, (i32x4_any*)p + i);
                    asm volatile("");
                } else {
                    ((i32x4_any*)p)[i] = a;
                }
            }
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = 0;
    }
    // nothing computed from these words before is kept: what is needed again is formed from them again, and the registers hold the words alone
    __device__ __forceinline__ void refresh() {
#pragma unroll
        for (int i = 0; i < W; ++i) asm volatile("" : "+v"(w[i]));
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

// f(f(a, b), ...) over groups of L lanes, the same in every lane (all lanes of the wave take part)
template <int CTRL> __device__ __forceinline__ float dpp(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, false)); }
template <int L, typename F> __device__ __forceinline__ float lanes_fold(float v, F&& f) {
    static_assert(L == 8 || L == 16 || L == 32 || L == 64, "lanes of a wave");
    v = f(v, dpp<0xB1>(v));    // lane ^ 1
    v = f(v, dpp<0x4E>(v));    // lane ^ 2
    v = f(v, dpp<0x141>(v));   // 7 - lane: the other four of eight
    if constexpr (L >= 16) v = f(v, dpp<0x140>(v));   // 15 - lane
    if constexpr (L >= 32) {   // rows of 16 lanes, then halves of 32, exchanged between two copies
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        const auto p = __builtin_amdgcn_permlane16_swap(b, b, false, false);
        const uint32_t x = p[0], y = p[1];
        v = f(__builtin_bit_cast(float, x), __builtin_bit_cast(float, y));
    }
    if constexpr (L >= 64) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        const auto p = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        const uint32_t x = p[0], y = p[1];
        v = f(__builtin_bit_cast(float, x), __builtin_bit_cast(float, y));
    }
    return v;
}
template <int L> __device__ __forceinline__ float lanes_sum(float v) { return lanes_fold<L>(v, [](float a, float b) { return a + b; }); }
// the same over a group of L threads: lanes of a wave, or waves of a workgroup, which meet in slot (two slots taken in turn need no other barrier)
template <int L, typename F> __device__ __forceinline__ float group_fold(float v, float* slot, F&& f) {
    if constexpr (L <= kWave) {
        return lanes_fold<L>(v, f);
    } else {
        v = lanes_fold<kWave>(v, f);
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
        __syncthreads();
        const float* own = slot + threadIdx.x / L * (L / kWave);
        float s = own[0];
#pragma unroll
        for (int i = 1; i < L / kWave; ++i) s = f(s, own[i]);
        return s;
    }
}
template <int L> __device__ __forceinline__ float group_sum(float v, float* slot) { return group_fold<L>(v, slot, [](float a, float b) { return a + b; }); }
template <int L> __device__ __forceinline__ float group_max(float v, float* slot) { return group_fold<L>(v, slot, [](float a, float b) { return fmaxf(a, b); }); }

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
// Rows in registers: a group of L threads (lanes of a wave, or waves of a workgroup) holds a row as K chunks of V values a thread, chunk k of thread l being number
// k * L + l.  The last chunk of a row whose length is no multiple of V ends with the row and overlaps the one before it: the values that both hold count once in sums and are
// stored twice, the same.  Threads beyond the last chunk hold that chunk too, count nothing and store nothing.  (The K of a length is the smallest: all but the last
// chunk of a thread are whole.)
constexpr int kThreads = 256;
template <int L> constexpr int threads_of() { return L <= kThreads ? kThreads : L; }

template <int L, int K, int V> struct RowPart {
    int at[K];      // first value of each chunk
    int skip;       // values at the start of chunk K - 1 that the chunk before it holds (V: all, nothing is stored)
    __device__ __forceinline__ RowPart(int l, int width) {
#pragma unroll
        for (int k = 0; k < K; ++k) at[k] = (k * L + l) * V;
        const int last = width - V;
        skip = at[K - 1] > last ? (at[K - 1] < width ? at[K - 1] - last : V) : 0;
        at[K - 1] = at[K - 1] > last ? last : at[K - 1];
    }
    __device__ __forceinline__ bool counts(int k, int i) const { return k < K - 1 || i >= skip; }
    __device__ __forceinline__ bool stores(int k) const { return k < K - 1 || skip < V; }
};

// calls f(L, K) as compile-time constants: the smallest group that holds `chunks` chunks, in waves' lanes first, then workgroups; false if none does
template <int A, int B> struct Shape { static constexpr int L = A, K = B; };
// TWO_WAVES: rows of up to 512 chunks by groups of 128 threads, four chunks each, rather than of 256, two each (layer norm's gradient of 65536 x 2048 values 148 us and 157, cross entropy of
// 20000 x 2001 in float32 57.8 and 54.5)
template <bool TWO_WAVES, typename F> bool with_shape(int chunks, F&& f) {
    bool done = false;
    auto take = [&](auto s) {
        if (!done && chunks <= decltype(s)::L * decltype(s)::K) {
            f(s);
            done = true;
        }
    };
    take(Shape<8, 1>{}); take(Shape<8, 2>{}); take(Shape<8, 3>{}); take(Shape<8, 4>{}); take(Shape<16, 3>{}); take(Shape<16, 4>{}); take(Shape<32, 3>{}); take(Shape<32, 4>{});
    take(Shape<64, 3>{}); take(Shape<64, 4>{}); take(Shape<128, 3>{}); take(std::conditional_t<TWO_WAVES, Shape<128, 4>, Shape<256, 2>>{}); take(Shape<256, 3>{}); take(Shape<256, 4>{}); take(Shape<512, 3>{}); take(Shape<512, 4>{});
    return done;
}
// the same for workgroups of 1024 threads
template <int K = 3, typename F> bool with_long_shape(int chunks, F&& f) {
    if constexpr (K > 16) {
        return false;
    } else {
        if (chunks > 1024 * K) return with_long_shape<K + 1>(chunks, f);
        f(Shape<1024, K>{});
        return true;
    }
}

template <int N> struct Int { static constexpr int value = N; };
// calls f with a null pointer of the C++ type behind a flashrnn_dtype_t / flashrnn_index_t
template <typename F> int with_io_type(int t, F&& f) { return t == FLASHRNN_BF16 ? f((__bf16*)nullptr) : f((float*)nullptr); }
template <typename F> int with_index_type(int t, F&& f) { return t == FLASHRNN_I64 ? f((int64_t*)nullptr) : f((int32_t*)nullptr); }

}  // namespace flashrnn
