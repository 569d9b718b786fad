// Cross entropy of rows of logits and its gradient (include/flashrnn.h).
//
// loss = log s + (top - x_t) and dx_j = f (exp(x_j - top) / s - [j = t]) with top the row's largest logit, s = sum exp(x_j - top), f = grad_scale * dloss; lse = top + log s where it is asked for (the loss
// does not go through lse, whose last place is that of the row's offset: beside logits of 30000 a loss of 0.0092 came out as 0.0098).  The call is
// bound by memory: a row is read once and its gradient written once, and in between it stays in registers as it lies in memory (16 bytes of it per word of four registers); the exponentials are
// formed twice rather than kept.  Sums are float32.  16384 x 50304 in bf16: 531 us, 6.2 TB/s; the loss alone 386, 4.3 TB/s.
#include "flashrnn_rows.h"

using namespace flashrnn;

namespace {

struct Problem {
    const void *logits, *targets;
    const float* dloss;
    float *loss, *lse;
    void* dlogits;
    size_t rows, stride, to_stride;
    int classes, index64;
    float scale;
};
__device__ __forceinline__ int64_t target_of(const Problem& p, size_t row) { return p.index64 ? ((const int64_t*)p.targets)[row] : ((const int32_t*)p.targets)[row]; }
// exp(x - top): the difference first, so that no finite logit overflows on the way
__device__ __forceinline__ float exp_below(float x, float top) { return fast_exp2((x - top) * kLog2e); }
// f exp(x - top), of the logits' type.  In float32 the rounding of d log2 e = y + (d - y ln 2) log2 e would leave classes 80 below the largest off by 62 units of 2^-24, so e^d = 2^y (1 + d - y ln 2), with ln 2
// in two parts.  (In the sum the plain form does: what it loses grows with the distance, and terms shrink with its exponential.  16384 x 128 in float32 4.95 us with the plain form in both, 5.18 so, 5.4 with the
// accurate one in both; 16384 x 32000 689, 697 and 733.)
constexpr float kLn2Hi = 0.693147182464599609375f, kLn2Lo = -1.904654299957767e-9f;
template <typename X> __device__ __forceinline__ float times_exp_below(float f, float x, float top) {
    if constexpr (sizeof(X) == 2) return f * exp_below(x, top);
    const float d = max_nan(x - top, -110.0f), y = d * kLog2e, p = f * fast_exp2(y);   // (-inf: p = 0)
    return fmaf(p, fmaf(-y, kLn2Lo, fmaf(-y, kLn2Hi, d)), p);
}

// Groups of L threads hold a row as K chunks of V values each, laid out as RowPart says.  Up to 7 chunks (57344 classes in bf16) the kernel keeps to 64 registers, so that a CU holds two
// workgroups of 1024 threads and one's loads and stores run beside the other's arithmetic: 16384 x 50304 in bf16 565 us, with one workgroup 653; eight chunks do not fit.
// STREAM: the gradient goes past the caches (536 us, 6.1 TB/s), decided when compiled because the 64 registers do not hold both stores.
template <typename X, int L, int K, bool STREAM>
__global__ __launch_bounds__(threads_of<L>(), L == 1024 && K <= 7 ? 8 : 1) void loss_rows_kernel(Problem p) {
    constexpr int V = 16 / sizeof(X), NT = threads_of<L>(), PER = NT / L;
    __shared__ float slots[2][NT / kWave];
    const int l = threadIdx.x % L;
    const RowPart<L, K, V> part(l, p.classes);
    for (size_t base = (size_t)blockIdx.x * PER + (L <= kWave ? threadIdx.x / kWave * (kWave / L) : 0); base < p.rows; base += (size_t)gridDim.x * PER) {
        const size_t row = base + (L <= kWave ? threadIdx.x % kWave / L : threadIdx.x / L);
        const bool there = row < p.rows;
        const int64_t t = there ? target_of(p, row) : -1;
        const bool counts = t >= 0 && t < p.classes;
        const int target = counts ? (int)t : -1;
        Chunk<X, V> raw[K];
        if (counts || (there && p.lse)) {   // (an ignored row is not read)
            const X* x = (const X*)p.logits + row * p.stride;
#pragma unroll
            for (int k = 0; k < K; ++k) raw[k].load(x + part.at[k]);
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) raw[k].clear();
        }
        float top = raw[0].get(0);   // fmaxf passes over NaN, which the sum then holds
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) top = fmaxf(top, raw[k].get(i));
        top = group_max<L>(top, slots[0]);
        if (top == -__builtin_inff()) top = 0.f;   // (nothing but -inf, whose terms are all 0 then, or NaN)
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            raw[k].refresh();
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float e = exp_below(raw[k].get(i), top);
                s += part.counts(k, i) ? e : 0.f;
            }
        }
        s = group_sum<L>(s, slots[1]);
        if (!there) continue;
        const float log_s = logf(s);
        if (l == 0) {
            if (p.lse) p.lse[row] = log_s + top;
            if (!counts) p.loss[row] = 0.f;
        }
        const float f = p.scale * (p.dloss ? p.dloss[row] : 1.f), fs = f / s;
        const bool zero = !counts || s == 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            raw[k].refresh();
            const int hit = target - part.at[k];   // the target's place in this chunk, where it holds it
            const bool holds = counts && hit >= 0 && hit < V;
            float g[V];
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] = zero ? 0.f : times_exp_below<X>(fs, raw[k].get(i), top);
            if (holds) {
                float x = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i == hit) {
                        x = raw[k].get(i);
                        if (!zero) g[i] -= f;
                    }
                if (part.stores(k)) p.loss[row] = s == 0.f ? __builtin_inff() : log_s + (top - x);
            }
            if (p.dlogits && part.stores(k)) {
                Chunk<X, V> c;
                c.put(g);
                c.store((X*)p.dlogits + row * p.to_stride + part.at[k], STREAM);
            }
        }
    }
}

// Rows that no group's registers hold (more than 131072 classes in bf16, 65536 in float32), and rows shorter than a chunk: read twice, the sum kept up with a running maximum.  3000 x 131072 in
// float32 744 us, 6.3 TB/s over two reads and a write; with no more workgroups than CUs, so that the second read could come from the last-level cache, 764.
template <typename X, int NT, bool STREAM>
__global__ __launch_bounds__(NT) void loss_long_kernel(Problem p) {
    constexpr int V = 16 / sizeof(X);
    __shared__ float slots[2][NT / kWave];
    const int whole = p.classes / V * V, tail = whole + threadIdx.x;   // (chunks, then a value each)
    for (size_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const X* x = (const X*)p.logits + row * p.stride;
        X* dx = (X*)p.dlogits + row * p.to_stride;
        const int64_t t = target_of(p, row);
        const bool counts = t >= 0 && t < p.classes;
        float top = -__builtin_inff(), s = 0.f;
        auto add = [&](float v, float m) { s += exp_below(v, m); };
        auto raise = [&](float m) {   // a larger maximum: what is there shrinks
            if (m > top) {
                s = s == 0.f ? 0.f : s * exp_below(top, m);
                top = m;
            }
        };
        for (int at = threadIdx.x * V; at < whole; at += NT * V) {
            Chunk<X, V> c;
            c.load(x + at);
            float m = c.get(0);
#pragma unroll
            for (int i = 1; i < V; ++i) m = fmaxf(m, c.get(i));
            raise(m);
#pragma unroll
            for (int i = 0; i < V; ++i) add(c.get(i), top == -__builtin_inff() ? 0.f : top);
        }
        if (tail < p.classes) {
            const float v = load_value(x + tail);
            raise(v);
            add(v, top == -__builtin_inff() ? 0.f : top);
        }
        float all = group_max<NT>(top, slots[0]);
        if (all == -__builtin_inff()) all = 0.f;
        s = top == -__builtin_inff() ? s : s * exp_below(top, all);   // (a thread without a maximum holds 0, or NaN)
        s = group_sum<NT>(s, slots[1]);
        const float log_s = logf(s), f = p.scale * (p.dloss ? p.dloss[row] : 1.f), fs = f / s;
        const bool zero = !counts || s == 0.f;
        if (threadIdx.x == 0) {
            if (p.lse) p.lse[row] = log_s + all;
            if (!counts) p.loss[row] = 0.f;
        }
        auto grad = [&](float v, int j) {
            const bool hit = counts && j == (int)t;
            if (hit) p.loss[row] = s == 0.f ? __builtin_inff() : log_s + (all - v);
            return zero ? 0.f : times_exp_below<X>(fs, v, all) - (hit ? f : 0.f);
        };
        if (!p.dlogits) {
            if (counts && threadIdx.x == 0) p.loss[row] = s == 0.f ? __builtin_inff() : log_s + (all - load_value(x + t));
            continue;
        }
        for (int at = threadIdx.x * V; at < whole; at += NT * V) {
            Chunk<X, V> c;
            c.load(x + at);
            float g[V];
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] = grad(c.get(i), at + i);
            c.put(g);
            c.store(dx + at, STREAM);
        }
        if (tail < p.classes) store_value(dx + tail, grad(load_value(x + tail), tail));
    }
}

}  // namespace

extern "C" int flashrnn_cross_entropy(const flashrnn_cross_entropy_desc_t* d, const void* logits, const void* targets, const void* dloss, void* loss, void* lse, void* dlogits,
                                      void* hip_stream) {
    if (!d) return FLASHRNN_ERR_NULL;
    if (d->rows < 0 || d->classes <= 0 || d->logits_stride < d->classes || (dlogits && d->dlogits_stride < d->classes)) return FLASHRNN_ERR_SHAPE;
    if (!is_io_type(d->io_dtype) || !is_index_type(d->index_dtype)) return FLASHRNN_ERR_SHAPE;
    if ((double)d->rows * (double)d->logits_stride > 1e18 || (dlogits && (double)d->rows * (double)d->dlogits_stride > 1e18)) return FLASHRNN_ERR_UNSUPPORTED;
    if (d->rows == 0) return FLASHRNN_OK;
    if (!logits || !targets || !loss) return FLASHRNN_ERR_NULL;
    const size_t e = type_size(d->io_dtype);
    if (!aligned_to(logits, e) || !aligned_to(dlogits, e) || !aligned_to(targets, type_size(d->index_dtype)) || !aligned_to(dloss, 4) || !aligned_to(loss, 4) || !aligned_to(lse, 4))
        return FLASHRNN_ERR_UNSUPPORTED;
    const size_t rows = (size_t)d->rows;
    const Problem p{logits, targets, (const float*)dloss, (float*)loss, (float*)lse, dlogits, rows, (size_t)d->logits_stride, (size_t)d->dlogits_stride, d->classes,
                    d->index_dtype == FLASHRNN_I64, d->grad_scale};
    const bool past_caches = rows * d->classes * e > kStreamBytes;
    const hipStream_t stream = (hipStream_t)hip_stream;
    return with_io_type(d->io_dtype, [&](auto* xt) {
        using X = std::remove_pointer_t<decltype(xt)>;
        constexpr int V = 16 / sizeof(X);
        int rc = FLASHRNN_OK;
        auto launch = [&](auto s) {
            constexpr int L = decltype(s)::L, K = decltype(s)::K, NT = threads_of<L>(), PER = NT / L;
            const dim3 grid(row_blocks((rows + PER - 1) / PER));
            if (past_caches) hipLaunchKernelGGL((loss_rows_kernel<X, L, K, true>), grid, dim3(NT), 0, stream, p);
            else hipLaunchKernelGGL((loss_rows_kernel<X, L, K, false>), grid, dim3(NT), 0, stream, p);
            rc = launch_status();
        };
        const int chunks = (d->classes + V - 1) / V;
        if (d->classes >= V && (with_shape<false>(chunks, launch) || with_long_shape(chunks, launch))) return rc;
        if (d->classes < V) hipLaunchKernelGGL((loss_long_kernel<X, kWave, false>), dim3(row_blocks(rows)), dim3(kWave), 0, stream, p);
        else if (past_caches) hipLaunchKernelGGL((loss_long_kernel<X, 1024, true>), dim3(row_blocks(rows)), dim3(1024), 0, stream, p);
        else hipLaunchKernelGGL((loss_long_kernel<X, 1024, false>), dim3(row_blocks(rows)), dim3(1024), 0, stream, p);
        return launch_status();
    });
}
