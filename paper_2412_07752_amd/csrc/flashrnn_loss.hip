// Cross entropy of rows of logits and its gradient (include/flashrnn.h).
#include "flashrnn_rows.h"

using namespace flashrnn;

namespace {

constexpr int kThreads = 256;

template <typename X, typename I>
__global__ __launch_bounds__(kThreads) void cross_entropy_kernel(size_t rows, int classes, size_t x_stride, size_t dx_stride, const X* logits, const I* __restrict__ targets,
                                                                 const float* __restrict__ dloss, float scale, float* __restrict__ loss, float* __restrict__ lse_out, X* dlogits) {
    __shared__ float lds[kThreads / kWave];
    for (size_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const X* x = logits + row * x_stride;
        const int64_t target = targets[row];
        const bool counts = target >= 0 && target < classes;
        // the largest logit; fmaxf passes over NaN, which the sum then holds
        float top = -__builtin_inff();
        for (int j = threadIdx.x; j < classes; j += kThreads) top = fmaxf(top, load_value(x + j));
        top = block_max<kThreads>(top, lds);
        if (top == -__builtin_inff()) top = 0.f;   // (nothing but -inf, whose terms are all 0 then, or NaN)
        float s = 0.f;
        for (int j = threadIdx.x; j < classes; j += kThreads) s += expf(load_value(x + j) - top);
        s = block_sum<kThreads>(s, lds);
        const float lse = logf(s) + top;
        if (threadIdx.x == 0) {
            loss[row] = !counts ? 0.f : s == 0.f ? __builtin_inff() : lse - load_value(x + target);
            if (lse_out) lse_out[row] = lse;
        }
        if (!dlogits) continue;
        __syncthreads();   // (thread 0 has read the target's logit, which an output in place overwrites)
        X* dx = dlogits + row * dx_stride;
        const float factor = scale * (dloss ? dloss[row] : 1.f);
        for (int j = threadIdx.x; j < classes; j += kThreads) {
            const float p = expf(load_value(x + j) - top) / s;
            store_value(dx + j, counts && s != 0.f ? factor * (p - (j == target ? 1.f : 0.f)) : 0.f);
        }
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
    return with_io_type(d->io_dtype, [&](auto* xt) {
        return with_index_type(d->index_dtype, [&](auto* it) {
            using X = std::remove_pointer_t<decltype(xt)>;
            using I = std::remove_pointer_t<decltype(it)>;
            hipLaunchKernelGGL((cross_entropy_kernel<X, I>), dim3(row_blocks((size_t)d->rows)), dim3(kThreads), 0, (hipStream_t)hip_stream, (size_t)d->rows, d->classes, (size_t)d->logits_stride,
                               (size_t)d->dlogits_stride, (const X*)logits, (const I*)targets, (const float*)dloss, d->grad_scale, (float*)loss, (float*)lse, (X*)dlogits);
            return launch_status();
        });
    });
}
