// Rows of activations, or output channels of a weight, as 8-bit whole numbers with a scale each.
#include "common.hpp"
#include "kernels.hpp"
#include "quant.hpp"

namespace meteora {

template <typename TX, int HELD>
__global__ __launch_bounds__(kQuantThreads) void quantize_rows_kernel(const TX* __restrict__ x, int d, int8_t* __restrict__ q,
                                                                      float* __restrict__ scale) {
    __shared__ float red[4];
    const size_t row = blockIdx.x;
    uint2* dst = reinterpret_cast<uint2*>(q + row * d);
    const float a = quantize_row<TX, HELD>(x + row * d, d / 8, red, [&](int i, uint2 v) { dst[i] = v; });
    if (threadIdx.x == 0) scale[row] = a / 127.f;
}

template <typename TX>
static hipError_t launch_quantize(const TX* x, int rows, int d, int8_t* q, float* scale, hipStream_t stream) {
    const int per_thread = ceil_div(d / 8, kQuantThreads);
    auto go = [&](auto kern) {
        kern<<<rows, kQuantThreads, 0, stream>>>(x, d, q, scale);
        return hipGetLastError();
    };
    if (per_thread <= 1) return go(&quantize_rows_kernel<TX, 1>);
    if (per_thread <= 2) return go(&quantize_rows_kernel<TX, 2>);
    if (per_thread <= 4) return go(&quantize_rows_kernel<TX, 4>);
    if (per_thread <= kQuantHeld) return go(&quantize_rows_kernel<TX, kQuantHeld>);
    return go(&quantize_rows_kernel<TX, 0>);
}

hipError_t launch_quantize_rows(const void* x, int rows, int d, bool bf16, int8_t* q, float* scale, hipStream_t stream) {
    return bf16 ? launch_quantize((const bf16_t*)x, rows, d, q, scale, stream)
                : launch_quantize((const float*)x, rows, d, q, scale, stream);
}

}  // namespace meteora
