// Rows of activations, or output channels of a weight, as 8-bit whole numbers with a scale each.
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"
#include "quant.hpp"

namespace meteora {

template <typename TX, int G, int HELD>
__global__ __launch_bounds__(kQuantThreads) void quantize_rows_kernel(const TX* __restrict__ x, int rows, int d,
                                                                      int8_t* __restrict__ q, float* __restrict__ scale) {
    __shared__ float red[4];
    const int row = (int)((blockIdx.x * (unsigned)kQuantThreads + threadIdx.x) / G);
    if (row >= rows) return;   // G = 256: never
    const TX* src = x + (size_t)row * d;
    uint2* dst = reinterpret_cast<uint2*>(q + (size_t)row * d);
    QuantRow<TX, G, HELD> r;
    r.load(src, d / 8);
    const float a = r.top(src, d / 8, red);
    r.store(src, d / 8, a, [&](int i, uint2 v) { dst[i] = v; });
    if ((threadIdx.x & (G - 1)) == 0) scale[row] = a / 127.f;
}

template <typename TX>
static hipError_t launch_quantize(const TX* x, int rows, int d, int8_t* q, float* scale, hipStream_t stream) {
    return quant_row_shape(d, rows >= 2048, [&](auto g, auto held) {
        constexpr int G = decltype(g)::value, HELD = decltype(held)::value;
        quantize_rows_kernel<TX, G, HELD><<<ceil_div(rows, kQuantThreads / G), kQuantThreads, 0, stream>>>(x, rows, d, q, scale);
        return hipGetLastError();
    });
}

hipError_t launch_quantize_rows(const void* x, int rows, int d, bool bf16, int8_t* q, float* scale, hipStream_t stream) {
    return bf16 ? launch_quantize((const bf16_t*)x, rows, d, q, scale, stream)
                : launch_quantize((const float*)x, rows, d, q, scale, stream);
}

}  // namespace meteora
