// Rows of activations, or output channels of a weight, as 4-bit values with block scales, and back.
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"
#include "quant_mx4.hpp"

namespace meteora {

// A wavefront takes a chunk of 512 inputs of a row at a time, 8 inputs a lane, a block to a quad of lanes.  A workgroup has 8 rows and two
// chunks of each, so that it writes whole lines of 128 bytes of scales, and a lane has 4 loads in flight.  Memory bounds it: 8192 x 4096 in bf16 16.7 us
// (5.1 TB/s), 4096 x 4096 8.5.
constexpr int kMxRows = 8, kMxCols = 2;

template <typename TX>
__global__ __launch_bounds__(256) void quantize_mx4_kernel(const TX* __restrict__ x, int rows, int d, int col_groups, uint8_t* __restrict__ q,
                                                           uint8_t* __restrict__ scale) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int group = blockIdx.x / col_groups, c0 = (blockIdx.x - group * col_groups) * kMxCols;
    const int chunks = mx4_chunks(d);
    Piece8<TX> p[2][kMxCols];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < kMxCols; ++c) {
            const int row = group * kMxRows + wave + h * 4, i = (c0 + c) * kMxChunk + lane * 8;
            p[h][c] = Piece8<TX>{};
            if (row < rows && i < d) p[h][c].load(x + (size_t)row * d + i);
        }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < kMxCols; ++c) {
            const int row = group * kMxRows + wave + h * 4, i = (c0 + c) * kMxChunk + lane * 8;
            const uint32_t E = mx4_exponent(p[h][c]);   // blocks past d are zeros: 0
            const uint32_t v = mx4_quantize8(p[h][c], E);
            if (row >= rows || c0 + c >= chunks) continue;
            if (i < d) *reinterpret_cast<uint32_t*>(q + ((size_t)row * d + i) / 2) = v;
            const int b = lane >> 2;
            if ((lane & 3) == 0) scale[((size_t)(c0 + c) * rows + row) * 16 + (b & 3) * 4 + (b >> 2)] = (uint8_t)E;
        }
}

hipError_t launch_quantize_mx4(const void* x, int rows, int d, bool bf16, uint8_t* q, uint8_t* scale, hipStream_t stream) {
    const int col_groups = ceil_div(mx4_chunks(d), kMxCols);
    const int64_t grid = (int64_t)ceil_div(rows, kMxRows) * col_groups;
    if (grid * 256 >= (int64_t)1 << 32) return hipErrorInvalidValue;
    if (bf16) quantize_mx4_kernel<<<(int)grid, 256, 0, stream>>>((const bf16_t*)x, rows, d, col_groups, q, scale);
    else quantize_mx4_kernel<<<(int)grid, 256, 0, stream>>>((const float*)x, rows, d, col_groups, q, scale);
    return hipGetLastError();
}

__device__ __forceinline__ uint32_t mx4_scale_byte(const uint8_t* scale, int rows, int row, int block) {
    return scale[((size_t)(block >> 4) * rows + row) * 16 + (block & 3) * 4 + ((block & 15) >> 2)];
}
__device__ __forceinline__ void store_values(bf16_t* dst, uint32_t q, float s) { *reinterpret_cast<u32x4*>(dst) = mx4_bf16x8(q, s); }
__device__ __forceinline__ void store_values(float* dst, uint32_t q, float s) {
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 1);
    const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 3);
    reinterpret_cast<f32x4*>(dst)[0] = f32x4{a[0], a[1], b[0], b[1]};
    reinterpret_cast<f32x4*>(dst)[1] = f32x4{c[0], c[1], e[0], e[1]};
}

// 8 values a lane, a chunk of 512 a wavefront, shared out as above: 4096 x 4096 8.0 us (5.3 TB/s).
template <typename TO>
__global__ __launch_bounds__(256) void dequantize_mx4_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ scale, int rows, int d,
                                                             int col_groups, TO* __restrict__ out) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int group = blockIdx.x / col_groups, c0 = (blockIdx.x - group * col_groups) * kMxCols;
    uint32_t v[2][kMxCols], E[2][kMxCols];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < kMxCols; ++c) {
            const int row = group * kMxRows + wave + h * 4, i = (c0 + c) * kMxChunk + lane * 8;
            v[h][c] = E[h][c] = 0;
            if (row < rows && i < d) {
                v[h][c] = *reinterpret_cast<const uint32_t*>(q + ((size_t)row * d + i) / 2);
                E[h][c] = mx4_scale_byte(scale, rows, row, i / kMxBlock);
            }
        }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < kMxCols; ++c) {
            const int row = group * kMxRows + wave + h * 4, i = (c0 + c) * kMxChunk + lane * 8;
            if (row < rows && i < d) store_values(out + (size_t)row * d + i, v[h][c], mx4_scale(E[h][c]));
        }
}

// out[d, rows].  A workgroup turns 64 rows of TD inputs: a thread takes 32 inputs of two neighbouring rows, whose values for one input are
// neighbours of the result, into LDS, from where they leave as 16-byte pieces of whole lines: 14336 x 4096 25 us (5.9 TB/s).
template <typename TO> constexpr int kTurnInputs = sizeof(TO) == 2 ? 256 : 128;
template <typename TO>
__global__ __launch_bounds__(kTurnInputs<TO>) void dequantize_mx4_turned_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ scale,
                                                                                int rows, int d, int row_groups, TO* __restrict__ out) {
    constexpr int TD = kTurnInputs<TO>, EB = sizeof(TO), LD = 64 * EB + 16;   // bytes of a row in LDS
    __shared__ __attribute__((aligned(16))) unsigned char turned[TD * LD];
    const int tid = threadIdx.x, r2 = tid & 31, piece = tid >> 5;   // TD / 32 pieces
    const int i0 = blockIdx.x / row_groups * TD, r0 = (blockIdx.x % row_groups) * 64;
    const int i = i0 + piece * 32;
    u32x4 v[2] = {};
    float s[2] = {};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = r0 + r2 * 2 + h;
        if (row < rows && i < d) {
            v[h] = *reinterpret_cast<const u32x4*>(q + ((size_t)row * d + i) / 2);
            s[h] = mx4_scale(mx4_scale_byte(scale, rows, row, i / kMxBlock));
        }
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        unsigned char* const at = turned + (piece * 32 + w * 8) * LD + r2 * 2 * EB;
        if constexpr (EB == 2) {
            const u32x4 a = mx4_bf16x8(v[0][w], s[0]), b = mx4_bf16x8(v[1][w], s[1]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                *reinterpret_cast<uint32_t*>(at + (2 * j) * LD) = __builtin_amdgcn_perm(b[j], a[j], 0x05040100u);
                *reinterpret_cast<uint32_t*>(at + (2 * j + 1) * LD) = __builtin_amdgcn_perm(b[j], a[j], 0x07060302u);
            }
        } else {
            float a[8], b[8];
            store_values(a, v[0][w], s[0]);
            store_values(b, v[1][w], s[1]);
#pragma unroll
            for (int j = 0; j < 8; ++j) *reinterpret_cast<float2*>(at + j * LD) = make_float2(a[j], b[j]);
        }
    }
    __syncthreads();
    constexpr int PPR = 64 * EB / 16;   // pieces per row of the result
#pragma unroll 4
    for (int p = tid; p < TD * PPR; p += TD) {
        const int r = p / PPR, c = p % PPR;
        const int col = r0 + c * (16 / EB);
        if (i0 + r >= d || col >= rows) continue;
        const u32x4 t = *reinterpret_cast<const u32x4*>(turned + r * LD + c * 16);
        *reinterpret_cast<u32x4*>(out + (size_t)(i0 + r) * rows + col) = t;   // rows % 8 == 0
    }
}

template <typename TO>
static hipError_t launch_dequantize(const uint8_t* q, const uint8_t* scale, int rows, int d, bool turned, TO* out, hipStream_t stream) {
    if (turned) {
        const int row_groups = ceil_div(rows, 64);
        const int64_t grid = (int64_t)ceil_div(d, kTurnInputs<TO>) * row_groups;
        if (grid * kTurnInputs<TO> >= (int64_t)1 << 32) return hipErrorInvalidValue;
        dequantize_mx4_turned_kernel<TO><<<(int)grid, kTurnInputs<TO>, 0, stream>>>(q, scale, rows, d, row_groups, out);
    } else {
        const int col_groups = ceil_div(mx4_chunks(d), kMxCols);
        const int64_t grid = (int64_t)ceil_div(rows, kMxRows) * col_groups;
        if (grid * 256 >= (int64_t)1 << 32) return hipErrorInvalidValue;
        dequantize_mx4_kernel<TO><<<(int)grid, 256, 0, stream>>>(q, scale, rows, d, col_groups, out);
    }
    return hipGetLastError();
}
hipError_t launch_dequantize_mx4(const uint8_t* q, const uint8_t* scale, int rows, int d, bool turned, bool bf16, void* out,
                                 hipStream_t stream) {
    return bf16 ? launch_dequantize(q, scale, rows, d, turned, (bf16_t*)out, stream)
                : launch_dequantize(q, scale, rows, d, turned, (float*)out, stream);
}

}  // namespace meteora
