// Layer norm over the rows of a tensor, one weight row for all of them or one per head, and its gradient (include/flashrnn.h).
//
// y = (x - mean) rstd w + b;  dx = rstd (g - E g - xh E(g xh)) with g = dy w, xh = (x - mean) rstd;  dw = sum dy xh, db = sum dy.  Both directions are bound by memory: x (and dy) are read once, y (or dx)
// is written once, and the row stays in registers between its sums; the mean first, then the squares around it, so that an offset costs no digits.  All sums are float32.  Measured:
// forward 65536 x 8 x 256 float32 states to bf16 141 us (5.7 TB/s), 65536 x 2048 bf16 91 us (5.9 TB/s); gradient 65536 x 8 x 256 199 us (5.4 TB/s), 16384 x 768 bf16 18.9 us (4.0 TB/s, 4 us of it the
// second kernel), up to 512 rows in one launch: 64 x 768 bf16 5.7 us.  Rows of fewer than 8 values, and of more than 16384 (bf16: 24576) forward or 12288 (all bf16: 16384) backward, take general kernels that read them several times, a value at a time
// (float32, 3000 x 30000 forward 1.6 TB/s, 20000 rows 1.7; 3000 x 16000 backward 1.6, 20000 rows 2.1).
#include "flashrnn_rows.h"

using namespace flashrnn;

namespace {

// Workgroups of a forward call: 65536 x 8 x 256 states (stored through the caches) take 161 us with 768 workgroups of 256 threads, 162 with 2048, 148 with 8192 and 160 with one row for
// every group of threads.
constexpr unsigned kMostThreads = 8192 * 256;
// ... and of a gradient, whose workgroups each leave partial sums of dweight and dbias: 16384 x 768 values in bf16 take 20.2 us with 256 workgroups of 256 threads, 18.6 with 512, 19.2 with 768
// and 20.0 with 1024; 65536 x 8 x 256 states 191, 197, 213 and 220, 65536 x 1200 in bf16 153, 100, 97 and 98.
constexpr unsigned kMostGradThreads = 512 * 256;
constexpr int kMaxStrips = 256;   // workgroups that add up the gradients of weight and bias, each over a strip of rows

// y may be x, and dx dy or x: a row is read, by the threads that hold it, before anything of it is written, and no pointer of the three is restricted.
struct Rows {
    long long x_stride;
    uint32_t count, per_outer;   // rows, and those of one outer block
    int groups, width;
};
__device__ __forceinline__ size_t x_offset(const Rows& r, uint32_t row) {
    const uint32_t o = row / r.per_outer;
    return (size_t)o * r.x_stride + (size_t)(row - o * r.per_outer) * r.width;
}

template <typename X, typename Y, typename P>
__global__ __launch_bounds__(kThreads) void layer_norm_fwd_kernel(Rows r, const X* x, const P* __restrict__ weight, const P* __restrict__ bias, Y* y,
                                                                  float* __restrict__ mean_out, float* __restrict__ rstd_out, float eps) {
    __shared__ float lds[kThreads / kWave];
    for (uint32_t row = blockIdx.x; row < r.count; row += gridDim.x) {
        const X* xr = x + x_offset(r, row);
        const int g = (int)(row % r.groups);
        float s = 0.f;
        for (int j = threadIdx.x; j < r.width; j += kThreads) s += load_value(xr + j);
        const float mean = block_sum<kThreads>(s, lds) / r.width;
        s = 0.f;
        for (int j = threadIdx.x; j < r.width; j += kThreads) {
            const float c = load_value(xr + j) - mean;
            s += c * c;
        }
        const float rstd = 1.0f / sqrtf(block_sum<kThreads>(s, lds) / r.width + eps);
        for (int j = threadIdx.x; j < r.width; j += kThreads) {
            float v = (load_value(xr + j) - mean) * rstd;
            if (weight) v *= load_value(weight + (size_t)g * r.width + j);
            if (bias) v += load_value(bias + (size_t)g * r.width + j);
            store_value(y + (size_t)row * r.width + j, v);
        }
        if (mean_out && threadIdx.x == 0) {
            mean_out[row] = mean;
            rstd_out[row] = rstd;
        }
    }
}

// Rows in registers, laid out as RowPart says, read once.  Groups take rows a fixed number apart, which is a multiple of `groups`, so that a thread's part of weight and bias
// stays in its registers; the next row's loads are on their way while this row is worked on.
template <typename X, int V, int L, int K>
__global__ __launch_bounds__(threads_of<L>()) void layer_norm_rows_kernel(Rows r, const X* x, const void* __restrict__ weight, const void* __restrict__ bias,
                                                                         bool params_bf16, void* y, bool y_bf16, bool stream, float* __restrict__ mean_out,
                                                                         float* __restrict__ rstd_out, float eps) {
    constexpr int NT = threads_of<L>(), PER = NT / L;   // groups of threads in a workgroup
    __shared__ float slots[2][NT / kWave];
    const int l = threadIdx.x % L;
    const uint32_t stride = gridDim.x * PER, first = blockIdx.x * PER + threadIdx.x / L;
    const uint32_t lead = blockIdx.x * PER + (L <= kWave ? threadIdx.x / kWave * (kWave / L) : 0);   // the first row of those that go through the loop together
    const RowPart<L, K, V> part(l, r.width);
    float w[K][V], b[K][V];
    const size_t own = (size_t)(first % r.groups) * r.width;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (weight) load_chunk<V>(weight, params_bf16, own + part.at[k], w[k]);
        else
#pragma unroll
            for (int i = 0; i < V; ++i) w[k][i] = 1.f;
        if (bias) load_chunk<V>(bias, params_bf16, own + part.at[k], b[k]);
        else
#pragma unroll
            for (int i = 0; i < V; ++i) b[k][i] = 0.f;
    }
    Chunk<X, V> raw[K];
    auto fetch = [&](uint32_t row) __attribute__((always_inline)) {
        const X* p = x + x_offset(r, row < r.count ? row : r.count - 1);
#pragma unroll
        for (int k = 0; k < K; ++k) raw[k].load(p + part.at[k]);
    };
    fetch(first);
    const float n = (float)r.width;
    for (uint32_t base = lead, row = first; base < r.count; base += stride, row += stride) {
        float v[K][V], s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[k][i] = raw[k].get(i);
                s += part.counts(k, i) ? v[k][i] : 0.f;
            }
        if (base + stride < r.count) fetch(row + stride);
        const float mean = group_sum<L>(s, slots[0]) / n;
        s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[k][i] -= mean;
                s += part.counts(k, i) ? v[k][i] * v[k][i] : 0.f;
            }
        const float rstd = 1.0f / sqrtf(group_sum<L>(s, slots[1]) / n + eps);
        if (row < r.count) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
#pragma unroll
                for (int i = 0; i < V; ++i) v[k][i] = v[k][i] * rstd * w[k][i] + b[k][i];
                if (part.stores(k)) store_chunk<V>(y, y_bf16, (size_t)row * r.width + part.at[k], v[k], stream);
            }
            if (mean_out && l == 0) {
                mean_out[row] = mean;
                rstd_out[row] = rstd;
            }
        }
    }
}

// The gradient, rows in registers as above: dx from the row's two sums, and every thread's part of dweight and dbias in its registers over all rows that its group takes.
// At the end the groups of a workgroup that share a row of the weights meet in LDS and their sum, in the order of the groups, is one row of partial sums; with more
// rows of weights than groups every group writes its own.  dweight, dbias: [strips][groups][width] each, a strip for every workgroup, or for every `groups` groups of threads; or null.
// COLUMNS, for few rows: every group of threads takes one row, for dx alone, and the first `column_blocks` workgroups add up dweight and dbias themselves, each kSumColumns columns over all rows.
constexpr int kSumColumns = 32;
template <typename X, typename Y, int NT>
__device__ __forceinline__ void sum_columns(const Rows& r, const Y* __restrict__ dy, const X* __restrict__ x, const float* __restrict__ mean_in, const float* __restrict__ rstd_in,
                                            float* __restrict__ dweight, float* __restrict__ dbias) {
    constexpr int V = 4, L = kSumColumns / V, kGroups = NT / L, kAhead = 4;
    __shared__ float lds[NT / kWave][L][2 * V];
    const int l = threadIdx.x % L, blocks = (r.width + kSumColumns - 1) / kSumColumns, g = blockIdx.x / blocks, from = (blockIdx.x - g * blocks) * kSumColumns + l * V;
    const int at = from < r.width - V ? from : r.width - V;   // (of columns that two lanes have, both write the same sums)
    const uint32_t tokens = r.count / r.groups;
    float s[2 * V] = {};
    for (uint32_t t = threadIdx.x / L; t < tokens; t += kAhead * kGroups) {
        Chunk<X, V> raw_x[kAhead];
        Chunk<Y, V> raw_dy[kAhead];
        float mean[kAhead], rstd[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t row = (t + u * kGroups < tokens ? t + u * kGroups : tokens - 1) * r.groups + g;
            raw_x[u].load(x + x_offset(r, row) + at);
            raw_dy[u].load(dy + (size_t)row * r.width + at);
            mean[u] = mean_in[row];
            rstd[u] = rstd_in[row];
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (t + u * kGroups < tokens)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    s[i] += raw_dy[u].get(i) * ((raw_x[u].get(i) - mean[u]) * rstd[u]);
                    s[V + i] += raw_dy[u].get(i);
                }
    }
#pragma unroll
    for (int o = L; o < kWave; o *= 2)
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) s[i] += __shfl_xor(s[i], o);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (lane < L)
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) lds[w][l][i] = s[i];
    __syncthreads();
    if (threadIdx.x >= L) return;
#pragma unroll
    for (int v = 1; v < NT / kWave; ++v)
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) s[i] += lds[v][l][i];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float* out = which ? dbias : dweight;
        if (!out) continue;
        Chunk<float, V> c;
#pragma unroll
        for (int i = 0; i < V; ++i) c.w[i] = __builtin_bit_cast(uint32_t, s[which * V + i]);
        c.store(out + (size_t)g * r.width + at);
    }
}
template <typename X, typename Y, int V, int L, int K, bool COLUMNS>
__global__ __launch_bounds__(threads_of<L>()) void layer_norm_grad_rows_kernel(uint32_t column_blocks, Rows r, const Y* dy, const X* x, const void* __restrict__ weight,
                                                                              bool weight_bf16, const float* __restrict__ mean_in, const float* __restrict__ rstd_in,
                                                                              void* dx, bool dx_bf16, bool stream, float* __restrict__ dweight, float* __restrict__ dbias) {
    constexpr int NT = threads_of<L>(), PER = NT / L;
    if (COLUMNS && blockIdx.x < column_blocks) return sum_columns<X, Y, NT>(r, dy, x, mean_in, rstd_in, dweight, dbias);
    __shared__ float slots[2][2][NT / kWave];
    const int l = threadIdx.x % L, group = threadIdx.x / L;
    const uint32_t block = COLUMNS ? blockIdx.x - column_blocks : blockIdx.x, stride = (COLUMNS ? gridDim.x - column_blocks : gridDim.x) * PER, first = block * PER + group;
    const uint32_t lead = block * PER + (L <= kWave ? threadIdx.x / kWave * (kWave / L) : 0);
    const RowPart<L, K, V> part(l, r.width);
    float w[K][V], dw[K][V], db[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (weight) load_chunk<V>(weight, weight_bf16, (size_t)(first % r.groups) * r.width + part.at[k], w[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!weight) w[k][i] = 1.f;
            dw[k][i] = db[k][i] = 0.f;
        }
    }
    Chunk<X, V> raw_x[K];
    Chunk<Y, V> raw_dy[K];
    float mean = 0.f, rstd = 0.f;
    auto fetch = [&](uint32_t row) __attribute__((always_inline)) {
        row = row < r.count ? row : r.count - 1;
        const X* p = x + x_offset(r, row);
        const Y* q = dy + (size_t)row * r.width;
        mean = mean_in[row];   // (ahead of the row: 65536 x 2048 values in bf16 148 us, behind it 154)
        rstd = rstd_in[row];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            raw_x[k].load(p + part.at[k]);
            raw_dy[k].load(q + part.at[k]);
        }
    };
    fetch(first);
    const float n = (float)r.width;
    int turn = 0;
    for (uint32_t base = lead, row = first; base < r.count; base += stride, row += stride, turn ^= 1) {
        float xh[K][V], g[K][V], a = 0.f, b = 0.f;
        const float scale = rstd;
        const bool there = row < r.count;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                xh[k][i] = (raw_x[k].get(i) - mean) * rstd;
                g[k][i] = raw_dy[k].get(i);
                if (!COLUMNS && there) {   // (of a chunk's values that another one holds too, the other one's sums are written)
                    dw[k][i] += g[k][i] * xh[k][i];
                    db[k][i] += g[k][i];
                }
                g[k][i] *= w[k][i];
                a += part.counts(k, i) ? g[k][i] : 0.f;
                b += part.counts(k, i) ? g[k][i] * xh[k][i] : 0.f;
            }
        if (base + stride < r.count) fetch(row + stride);
        if constexpr (L <= kWave) {
            a = lanes_sum<L>(a);
            b = lanes_sum<L>(b);
        } else {   // (both sums behind one barrier; the slots alternate)
            a = lanes_sum<kWave>(a);
            b = lanes_sum<kWave>(b);
            if ((threadIdx.x & 63) == 0) {
                slots[turn][0][threadIdx.x >> 6] = a;
                slots[turn][1][threadIdx.x >> 6] = b;
            }
            __syncthreads();
            const int own = group * (L / kWave);
            a = slots[turn][0][own];
            b = slots[turn][1][own];
#pragma unroll
            for (int i = 1; i < L / kWave; ++i) {
                a += slots[turn][0][own + i];
                b += slots[turn][1][own + i];
            }
        }
        a /= n;
        b /= n;
        if (there) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
#pragma unroll
                for (int i = 0; i < V; ++i) g[k][i] = scale * (g[k][i] - a - xh[k][i] * b);
                if (part.stores(k)) store_chunk<V>(dx, dx_bf16, (size_t)row * r.width + part.at[k], g[k], stream);
            }
        }
    }
    if (COLUMNS || (!dweight && !dbias)) return;
    __shared__ float merge[PER > 1 && !COLUMNS ? 2 * NT * K * V : 1];
    if (PER > 1 && r.groups <= PER) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                merge[(k * V + i) * NT + threadIdx.x] = dw[k][i];
                merge[((K + k) * V + i) * NT + threadIdx.x] = db[k][i];
            }
        __syncthreads();
        // every thread some of the sums: a chunk of one thread of a group, or, where these are fewer than the threads, a value of one
        constexpr int N = 2 * L * K >= NT ? V : 1, kEach = L * K * V / N;
        const int half = r.groups * kEach;
        for (int o = threadIdx.x; o < 2 * half; o += NT) {
            const int which = o >= half, rest = o - (which ? half : 0), row = rest / kEach, of = rest % L, value = rest % kEach / L * N, begin = (value / V * L + of) * V;
            float* out = which ? dbias : dweight;
            if (!out || begin >= r.width) continue;
            const float* from = merge + (which * K * V + value) * NT + of;
            float sum[N] = {};
            for (int g = row; g < PER; g += r.groups)
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] += from[i * NT + g * L];
            const uint32_t to = blockIdx.x * r.groups + (r.groups == 1 ? 0 : (blockIdx.x * PER + row) % r.groups);
            out += (size_t)to * r.width + (begin < r.width - V ? begin : r.width - V) + value % V;
            if constexpr (N == V) {
                Chunk<float, V> c;
                c.put(sum);
                c.store(out);
            } else {
                *out = sum[0];
            }
        }
        return;
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float(&v)[K][V] = which ? db : dw;
        float* out = which ? dbias : dweight;
        if (!out) continue;
        out += (size_t)first * r.width;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (part.stores(k)) {
                Chunk<float, V> c;
                c.put(v[k]);
                c.store(out + part.at[k]);
            }
    }
}

// dweight and dbias from partial sums [dweight, dbias][strips][columns]: a wave adds up every kSumWaves-th strip of 64 columns, in order, then the waves meet
constexpr int kSumWaves = 16, kSumAhead = 8;   // (loads on their way)
__global__ __launch_bounds__(kSumWaves * kWave) void layer_norm_sum_strips_kernel(const float* __restrict__ part, size_t columns, int strips, float* __restrict__ dweight,
                                                                                 float* __restrict__ dbias) {
    __shared__ float lds[kSumWaves][kWave];
    float* out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const size_t col = (size_t)blockIdx.x * kWave + lane;
    const float* p = part + (size_t)blockIdx.y * strips * columns + (col < columns ? col : columns - 1);
    float s = 0.f;
    int i = w;
    for (; i + (kSumAhead - 1) * kSumWaves < strips; i += kSumAhead * kSumWaves) {
        float v[kSumAhead];
#pragma unroll
        for (int u = 0; u < kSumAhead; ++u) v[u] = p[(size_t)(i + u * kSumWaves) * columns];
#pragma unroll
        for (int u = 0; u < kSumAhead; ++u) s += v[u];
    }
    for (; i < strips; i += kSumWaves) s += p[(size_t)i * columns];
    lds[w][lane] = s;
    __syncthreads();
    if (w == 0 && col < columns) {
        for (int u = 1; u < kSumWaves; ++u) s += lds[u][lane];
        out[col] = s;
    }
}

// workgroups of PER groups of threads each: at most `most`, and a number that keeps a group's rows on one row of the weights
inline size_t lcm_of(size_t a, size_t b) {
    size_t x = a, y = b;
    while (y) {
        const size_t t = x % y;
        x = y;
        y = t;
    }
    return a / x * b;
}
inline unsigned blocks_for(size_t rows, int per, int groups, unsigned most) {
    const size_t want = (rows + per - 1) / per, unit = lcm_of(groups, per) / per;
    if (want <= most) return (unsigned)want;
    if (unit > (1u << 20)) return 0;   // (a dispatch holds fewer than 2^32 threads)
    const size_t blocks = most < unit ? unit : most / unit * unit;
    return (unsigned)(blocks < want ? blocks : want);
}

// Up to so many rows for every row of the weights, dweight and dbias come from the same launch, which reads x and dy twice: 64 rows of 768 values in bf16 5.5 us and, from partial sums, 9.0; 512 of 768 5.7
// and 9.1; 512 of 2048 7.8 and 9.3; 256 x 16 heads of 256 6.4 and 18.6; but 1024 of 1024 in float32 14.2 and 8.2.
constexpr size_t kColumnsRows = 512, kMostBlocks = 65536;
// launch of the gradient with rows in registers; blocks = 0: none
struct GradPlan {
    unsigned blocks;
    size_t sum_rows;   // rows of partial sums
};
inline GradPlan grad_plan(const Rows& r, int per, int threads) {
    GradPlan p{blocks_for(r.count, per, r.groups, kMostGradThreads / threads), 0};
    if (r.groups > per) {   // whole strips: workgroups beyond the rows write zeros
        const size_t unit = lcm_of(r.groups, per) / per;
        p.blocks = unit > (1u << 20) ? 0 : (unsigned)((p.blocks + unit - 1) / unit * unit);
    }
    if ((size_t)r.groups * r.width > (1u << 27)) p.blocks = 0;   // (a dispatch holds fewer than 2^32 threads, the sum's too)
    p.sum_rows = (size_t)p.blocks * (r.groups <= per ? r.groups : per);
    return p;
}

template <typename X, typename Y, typename DX, typename P>
__global__ __launch_bounds__(kThreads) void layer_norm_dx_kernel(Rows r, const Y* dy, const X* x, const P* __restrict__ weight,
                                                                 const float* __restrict__ mean_in, const float* __restrict__ rstd_in, DX* dx) {
    __shared__ float lds[kThreads / kWave];
    for (uint32_t row = blockIdx.x; row < r.count; row += gridDim.x) {
        const X* xr = x + x_offset(r, row);
        const Y* dyr = dy + (size_t)row * r.width;
        const P* w = weight ? weight + (size_t)(row % r.groups) * r.width : nullptr;
        const float mean = mean_in[row], rstd = rstd_in[row];
        float a = 0.f, b = 0.f;
        for (int j = threadIdx.x; j < r.width; j += kThreads) {
            const float g = load_value(dyr + j) * (w ? load_value(w + j) : 1.0f);
            a += g;
            b += g * ((load_value(xr + j) - mean) * rstd);
        }
        a = block_sum<kThreads>(a, lds) / r.width;
        b = block_sum<kThreads>(b, lds) / r.width;
        for (int j = threadIdx.x; j < r.width; j += kThreads) {
            const float g = load_value(dyr + j) * (w ? load_value(w + j) : 1.0f);
            store_value(dx + (size_t)row * r.width + j, rstd * (g - a - (load_value(xr + j) - mean) * rstd * b));
        }
    }
}

// partial sums of dweight and dbias: workgroup (column block, strip) adds the rows strip, strip + strips, ... of every group
template <typename X, typename Y>
__global__ __launch_bounds__(kThreads) void layer_norm_dparam_kernel(Rows r, size_t tokens, const Y* __restrict__ dy, const X* __restrict__ x, const float* __restrict__ mean_in,
                                                                     const float* __restrict__ rstd_in, float* __restrict__ part) {
    const size_t columns = (size_t)r.groups * r.width, col = (size_t)blockIdx.x * kThreads + threadIdx.x;
    if (col >= columns) return;
    const int g = (int)(col / r.width), j = (int)(col % r.width);
    float dw = 0.f, db = 0.f;
    for (size_t t = blockIdx.y; t < tokens; t += gridDim.y) {
        const uint32_t row = (uint32_t)t * r.groups + g;
        const float d = load_value(dy + (size_t)row * r.width + j);
        dw += d * ((load_value(x + x_offset(r, row) + j) - mean_in[row]) * rstd_in[row]);
        db += d;
    }
    float* p = part + (size_t)blockIdx.y * 2 * columns;
    p[col] = dw;
    p[columns + col] = db;
}

__global__ __launch_bounds__(kThreads) void layer_norm_sum_kernel(const float* __restrict__ part, size_t columns, int strips, float* __restrict__ dweight, float* __restrict__ dbias) {
    const size_t col = (size_t)blockIdx.x * kThreads + threadIdx.x;
    if (col >= 2 * columns) return;
    float s = 0.f;
    for (int i = 0; i < strips; ++i) s += part[(size_t)i * 2 * columns + col];
    float* out = col < columns ? dweight : dbias;
    if (out) out[col < columns ? col : col - columns] = s;
}

int check_desc(const flashrnn_layer_norm_desc_t* d) {
    if (!d) return FLASHRNN_ERR_NULL;
    if (d->rows_outer < 0 || d->rows_inner < 0 || d->x_stride < 0 || d->groups <= 0 || d->width <= 0 || !(d->eps >= 0.f)) return FLASHRNN_ERR_SHAPE;
    if (!is_io_type(d->x_dtype) || !is_io_type(d->io_dtype) || !is_io_type(d->dx_dtype) || !is_io_type(d->param_dtype)) return FLASHRNN_ERR_SHAPE;
    // rows below 2^31 (one workgroup each at most), every offset in bytes below 2^62
    const double rows = (double)d->rows_outer * (double)d->rows_inner * d->groups, extent = (double)d->rows_outer * (double)d->x_stride + rows * d->width;
    if (rows > 2147483647.0 || extent > 1e18 || (double)d->groups * d->width > 1073741824.0) return FLASHRNN_ERR_UNSUPPORTED;
    return FLASHRNN_OK;
}
Rows rows_of(const flashrnn_layer_norm_desc_t* d) {
    const size_t per_outer = (size_t)d->rows_inner * d->groups;   // (both below 2^31, or there are no rows)
    return Rows{d->x_stride, (uint32_t)(d->rows_outer * per_outer), (uint32_t)per_outer, d->groups, d->width};
}
int strips_of(const flashrnn_layer_norm_desc_t* d) {
    const size_t tokens = (size_t)d->rows_outer * d->rows_inner;
    return tokens < kMaxStrips ? (tokens ? (int)tokens : 1) : kMaxStrips;
}

// Calls f(X*, Y*, V, shape) for a gradient whose rows fit in registers.  Chunks of four values also in bf16, as long as a workgroup's registers hold the row: with eight the sums of
// dweight and dbias leave a SIMD one or two waves (16384 x 768 values 18.6 us and 21.0, 65536 x 256 25 and 32, 65536 x 2048 148 and 152).
template <typename F> void with_grad_shape(const flashrnn_layer_norm_desc_t* d, F&& f) {
    if (d->width < 8) return;
    with_io_type(d->x_dtype, [&](auto* xt) {
        return with_io_type(d->io_dtype, [&](auto* yt) {
            if (with_shape<true>((d->width + 3) / 4, [&](auto s) { f(xt, yt, Int<4>{}, s); })) return 0;
            // rows of more than 8192 values
            if constexpr (sizeof(*xt) == 2 && sizeof(*yt) == 2) {
                const int chunks = (d->width + 7) / 8;
                if (chunks <= 512 * 3) f(xt, yt, Int<8>{}, Shape<512, 3>{});
                else if (chunks <= 512 * 4) f(xt, yt, Int<8>{}, Shape<512, 4>{});
            } else {
                if (d->width <= 1024 * 3 * 4) f(xt, yt, Int<4>{}, Shape<1024, 3>{});
            }
            return 0;
        });
    });
}

}  // namespace

extern "C" {

size_t flashrnn_layer_norm_workspace_bytes(const flashrnn_layer_norm_desc_t* d) {
    if (check_desc(d) != FLASHRNN_OK) return 0;
    size_t rows = (size_t)strips_of(d) * d->groups;
    with_grad_shape(d, [&](auto, auto, auto, auto s) {
        constexpr int NT = threads_of<decltype(s)::L>();
        const GradPlan p = grad_plan(rows_of(d), NT / decltype(s)::L, NT);
        if (p.sum_rows) rows = p.sum_rows;
    });
    return (rows * 2 * d->width * sizeof(float) + 255) / 256 * 256;
}

int flashrnn_layer_norm_fwd(const flashrnn_layer_norm_desc_t* d, const void* x, const void* weight, const void* bias, void* y, void* mean, void* rstd, void* hip_stream) {
    const int rc = check_desc(d);
    if (rc != FLASHRNN_OK) return rc;
    const Rows r = rows_of(d);
    const size_t rows = r.count;
    if (rows == 0) return FLASHRNN_OK;
    if (!x || !y || (mean == nullptr) != (rstd == nullptr)) return FLASHRNN_ERR_NULL;
    if (!aligned_to(x, type_size(d->x_dtype)) || !aligned_to(y, type_size(d->io_dtype)) || !aligned_to(weight, type_size(d->param_dtype)) ||
        !aligned_to(bias, type_size(d->param_dtype)) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return FLASHRNN_ERR_UNSUPPORTED;
    int status = FLASHRNN_OK;
    bool taken = false;
    if (d->width >= 8) with_io_type(d->x_dtype, [&](auto* xt) {
        using X = std::remove_pointer_t<decltype(xt)>;
        constexpr int V = 16 / sizeof(X);
        const int chunks = (d->width + V - 1) / V;
        auto launch = [&](auto s) {
            constexpr int L = decltype(s)::L, K = decltype(s)::K, NT = threads_of<L>();
            const unsigned blocks = blocks_for(rows, NT / L, d->groups, kMostThreads / NT);
            if (!blocks) return;
            taken = true;
            hipLaunchKernelGGL((layer_norm_rows_kernel<X, V, L, K>), dim3(blocks), dim3(NT), 0, (hipStream_t)hip_stream, r, (const X*)x, weight, bias,
                               d->param_dtype == FLASHRNN_BF16, y, d->io_dtype == FLASHRNN_BF16, rows * d->width * type_size(d->io_dtype) > kStreamBytes, (float*)mean, (float*)rstd, d->eps);
            status = launch_status();
        };
        if (!with_shape<true>(chunks, launch)) {   // rows that a workgroup of 1024 threads holds
            if (chunks <= 1024 * 3) launch(Shape<1024, 3>{});
            else if (V == 4 && chunks <= 1024 * 4) launch(Shape<1024, V == 4 ? 4 : 3>{});
        }
        return 0;
    });
    if (taken) return status;
    return with_io_type(d->x_dtype, [&](auto* xt) {
        return with_io_type(d->io_dtype, [&](auto* yt) {
            return with_io_type(d->param_dtype, [&](auto* pt) {
                using X = std::remove_pointer_t<decltype(xt)>;
                using Y = std::remove_pointer_t<decltype(yt)>;
                using P = std::remove_pointer_t<decltype(pt)>;
                hipLaunchKernelGGL((layer_norm_fwd_kernel<X, Y, P>), dim3(row_blocks(rows)), dim3(kThreads), 0, (hipStream_t)hip_stream, r, (const X*)x, (const P*)weight,
                                   (const P*)bias, (Y*)y, (float*)mean, (float*)rstd, d->eps);
                return launch_status();
            });
        });
    });
}

int flashrnn_layer_norm_bwd(const flashrnn_layer_norm_desc_t* d, const void* dy, const void* x, const void* weight, const void* mean, const void* rstd, void* dx, void* dweight,
                            void* dbias, void* workspace, void* hip_stream) {
    int rc = check_desc(d);
    if (rc != FLASHRNN_OK) return rc;
    const Rows r = rows_of(d);
    const size_t rows = r.count, columns = (size_t)d->groups * d->width, tokens = rows / d->groups;
    if (rows && (!dy || !x || !mean || !rstd || !dx)) return FLASHRNN_ERR_NULL;
    const bool params = dweight || dbias;
    if (params && (!workspace || !aligned_to(workspace, 256))) return FLASHRNN_ERR_WORKSPACE;
    if (!aligned_to(x, type_size(d->x_dtype)) || !aligned_to(dy, type_size(d->io_dtype)) || !aligned_to(dx, type_size(d->dx_dtype)) ||
        !aligned_to(weight, type_size(d->param_dtype)) || !aligned_to(mean, 4) || !aligned_to(rstd, 4) || !aligned_to(dweight, 4) || !aligned_to(dbias, 4))
        return FLASHRNN_ERR_UNSUPPORTED;
    const hipStream_t stream = (hipStream_t)hip_stream;
    bool taken = false;
    int strips = 0;
    if (rows) with_grad_shape(d, [&](auto* xt, auto* yt, auto v, auto s) {
        using X = std::remove_pointer_t<decltype(xt)>;
        using Y = std::remove_pointer_t<decltype(yt)>;
        constexpr int L = decltype(s)::L, K = decltype(s)::K, NT = threads_of<L>();
        const size_t column_blocks = d->groups * (((size_t)d->width + kSumColumns - 1) / kSumColumns);
        if (params && dx != dy && dx != x && tokens <= kColumnsRows && rows <= kMostBlocks && column_blocks <= kMostBlocks) {   // (in place nothing can be read twice)
            taken = true;
            strips = 1;
            hipLaunchKernelGGL((layer_norm_grad_rows_kernel<X, Y, decltype(v)::value, L, K, true>), dim3((unsigned)(column_blocks + (rows + NT / L - 1) / (NT / L))), dim3(NT), 0, stream,
                               (uint32_t)column_blocks, r, (const Y*)dy, (const X*)x, weight, d->param_dtype == FLASHRNN_BF16, (const float*)mean, (const float*)rstd, dx,
                               d->dx_dtype == FLASHRNN_BF16, rows * d->width * type_size(d->dx_dtype) > kStreamBytes, (float*)dweight, (float*)dbias);
            rc = launch_status();
            return;
        }
        const GradPlan p = grad_plan(r, NT / L, NT);
        if (!p.blocks) return;
        taken = true;
        strips = (int)(p.sum_rows / r.groups);
        hipLaunchKernelGGL((layer_norm_grad_rows_kernel<X, Y, decltype(v)::value, L, K, false>), dim3(p.blocks), dim3(NT), 0, stream, 0u, r, (const Y*)dy, (const X*)x, weight,
                           d->param_dtype == FLASHRNN_BF16, (const float*)mean, (const float*)rstd, dx, d->dx_dtype == FLASHRNN_BF16,
                           rows * d->width * type_size(d->dx_dtype) > kStreamBytes, strips == 1 ? (float*)dweight : params ? (float*)workspace : nullptr,
                           strips == 1 ? (float*)dbias : params ? (float*)workspace + p.sum_rows * d->width : nullptr);
        rc = launch_status();
    });
    if (taken) {
        if (rc != FLASHRNN_OK || !params || strips == 1) return rc;
        hipLaunchKernelGGL(layer_norm_sum_strips_kernel, dim3((unsigned)((columns + kWave - 1) / kWave), 2), dim3(kSumWaves * kWave), 0, stream, (const float*)workspace, columns,
                           strips, (float*)dweight, (float*)dbias);
        return launch_status();
    }
    const unsigned column_blocks = (unsigned)((columns + kThreads - 1) / kThreads);
    rc = with_io_type(d->x_dtype, [&](auto* xt) {
        return with_io_type(d->io_dtype, [&](auto* yt) {
            using X = std::remove_pointer_t<decltype(xt)>;
            using Y = std::remove_pointer_t<decltype(yt)>;
            if (params) {
                hipLaunchKernelGGL((layer_norm_dparam_kernel<X, Y>), dim3(column_blocks, strips_of(d)), dim3(kThreads), 0, stream, r, tokens, (const Y*)dy, (const X*)x,
                                   (const float*)mean, (const float*)rstd, (float*)workspace);
                if (const int e = launch_status()) return e;
            }
            if (rows == 0) return (int)FLASHRNN_OK;
            return with_io_type(d->dx_dtype, [&](auto* dt) {
                return with_io_type(d->param_dtype, [&](auto* pt) {
                    using DX = std::remove_pointer_t<decltype(dt)>;
                    using P = std::remove_pointer_t<decltype(pt)>;
                    hipLaunchKernelGGL((layer_norm_dx_kernel<X, Y, DX, P>), dim3(row_blocks(rows)), dim3(kThreads), 0, stream, r, (const Y*)dy, (const X*)x, (const P*)weight,
                                       (const float*)mean, (const float*)rstd, (DX*)dx);
                    return launch_status();
                });
            });
        });
    });
    if (rc != FLASHRNN_OK || !params) return rc;
    hipLaunchKernelGGL(layer_norm_sum_kernel, dim3((unsigned)((2 * columns + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, (const float*)workspace, columns, strips_of(d),
                       (float*)dweight, (float*)dbias);
    return launch_status();
}

}  // extern "C"
