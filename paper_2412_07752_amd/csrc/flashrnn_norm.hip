// Layer norm over the rows of a tensor, one weight row for all of them or one per head, and its gradient (include/flashrnn.h).
#include "flashrnn_rows.h"

using namespace flashrnn;

namespace {

constexpr int kThreads = 256;
constexpr int kMaxStrips = 256;   // workgroups that add up the gradients of weight and bias, each over a strip of rows

struct Rows {
    long long inner, x_stride;
    int groups, width;
};
__device__ __forceinline__ size_t x_offset(const Rows& r, size_t row) {
    const size_t per_outer = (size_t)r.inner * r.groups;
    return row / per_outer * r.x_stride + row % per_outer * r.width;
}

template <typename X, typename Y, typename P>
__global__ __launch_bounds__(kThreads) void layer_norm_fwd_kernel(Rows r, size_t rows, const X* __restrict__ x, const P* __restrict__ weight, const P* __restrict__ bias, Y* __restrict__ y,
                                                                  float* __restrict__ mean_out, float* __restrict__ rstd_out, float eps) {
    __shared__ float lds[kThreads / kWave];
    for (size_t row = blockIdx.x; row < rows; row += gridDim.x) {
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
            store_value(y + row * r.width + j, v);
        }
        if (mean_out && threadIdx.x == 0) {
            mean_out[row] = mean;
            rstd_out[row] = rstd;
        }
    }
}

template <typename X, typename Y, typename DX, typename P>
__global__ __launch_bounds__(kThreads) void layer_norm_dx_kernel(Rows r, size_t rows, const Y* __restrict__ dy, const X* __restrict__ x, const P* __restrict__ weight,
                                                                 const float* __restrict__ mean_in, const float* __restrict__ rstd_in, DX* __restrict__ dx) {
    __shared__ float lds[kThreads / kWave];
    for (size_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const X* xr = x + x_offset(r, row);
        const Y* dyr = dy + row * r.width;
        const P* w = weight ? weight + row % r.groups * r.width : nullptr;
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
            store_value(dx + row * r.width + j, rstd * (g - a - (load_value(xr + j) - mean) * rstd * b));
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
        const size_t row = t * r.groups + g;
        const float d = load_value(dy + row * r.width + j);
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
    if (rows > 2147483647.0 || extent > 1e18 || (double)d->groups * d->width > 2147483647.0) return FLASHRNN_ERR_UNSUPPORTED;
    return FLASHRNN_OK;
}
size_t rows_of(const flashrnn_layer_norm_desc_t* d) { return (size_t)d->rows_outer * d->rows_inner * d->groups; }
int strips_of(const flashrnn_layer_norm_desc_t* d) {
    const size_t tokens = (size_t)d->rows_outer * d->rows_inner;
    return tokens < kMaxStrips ? (tokens ? (int)tokens : 1) : kMaxStrips;
}

}  // namespace

extern "C" {

size_t flashrnn_layer_norm_workspace_bytes(const flashrnn_layer_norm_desc_t* d) {
    if (check_desc(d) != FLASHRNN_OK) return 0;
    const size_t bytes = (size_t)strips_of(d) * 2 * d->groups * d->width * sizeof(float);
    return (bytes + 255) / 256 * 256;
}

int flashrnn_layer_norm_fwd(const flashrnn_layer_norm_desc_t* d, const void* x, const void* weight, const void* bias, void* y, void* mean, void* rstd, void* hip_stream) {
    const int rc = check_desc(d);
    if (rc != FLASHRNN_OK) return rc;
    const size_t rows = rows_of(d);
    if (rows == 0) return FLASHRNN_OK;
    if (!x || !y || (mean == nullptr) != (rstd == nullptr)) return FLASHRNN_ERR_NULL;
    if (!aligned_to(x, type_size(d->x_dtype)) || !aligned_to(y, type_size(d->io_dtype)) || !aligned_to(weight, type_size(d->param_dtype)) ||
        !aligned_to(bias, type_size(d->param_dtype)) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return FLASHRNN_ERR_UNSUPPORTED;
    const Rows r{d->rows_inner, d->x_stride, d->groups, d->width};
    return with_io_type(d->x_dtype, [&](auto* xt) {
        return with_io_type(d->io_dtype, [&](auto* yt) {
            return with_io_type(d->param_dtype, [&](auto* pt) {
                using X = std::remove_pointer_t<decltype(xt)>;
                using Y = std::remove_pointer_t<decltype(yt)>;
                using P = std::remove_pointer_t<decltype(pt)>;
                hipLaunchKernelGGL((layer_norm_fwd_kernel<X, Y, P>), dim3(row_blocks(rows)), dim3(kThreads), 0, (hipStream_t)hip_stream, r, rows, (const X*)x, (const P*)weight,
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
    const size_t rows = rows_of(d), columns = (size_t)d->groups * d->width, tokens = rows / d->groups;
    if (rows && (!dy || !x || !mean || !rstd || !dx)) return FLASHRNN_ERR_NULL;
    const bool params = dweight || dbias;
    if (params && (!workspace || !aligned_to(workspace, 256))) return FLASHRNN_ERR_WORKSPACE;
    if (!aligned_to(x, type_size(d->x_dtype)) || !aligned_to(dy, type_size(d->io_dtype)) || !aligned_to(dx, type_size(d->dx_dtype)) ||
        !aligned_to(weight, type_size(d->param_dtype)) || !aligned_to(mean, 4) || !aligned_to(rstd, 4) || !aligned_to(dweight, 4) || !aligned_to(dbias, 4))
        return FLASHRNN_ERR_UNSUPPORTED;
    const Rows r{d->rows_inner, d->x_stride, d->groups, d->width};
    const hipStream_t stream = (hipStream_t)hip_stream;
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
                    hipLaunchKernelGGL((layer_norm_dx_kernel<X, Y, DX, P>), dim3(row_blocks(rows)), dim3(kThreads), 0, stream, r, rows, (const Y*)dy, (const X*)x, (const P*)weight,
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
