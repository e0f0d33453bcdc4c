// Rows as 8-bit whole numbers with one scale each (device side, shared by quant.hip and sort.hip):
//     a = max_i |x_i|,   q_i = 127 x_i / a rounded to the nearest whole number, halves to the even one,   scale = a / 127.
// The quotient is the exact one's rounding, not an approximation's: x_i = a / 2 is 63.5, and bf16 rows hold such values often (one
// in about 256 of the elements of an octave), so whether a half is seen as one decides a whole step of the result.
#pragma once
#include "common.hpp"

namespace meteora {

constexpr int kQuantThreads = 256;   // threads that share a row
constexpr int kQuantHeld = 8;        // pieces of 8 elements that a thread holds between the two passes: rows of up to 16384 elements

// 8 consecutive elements as they are stored
template <typename TX> struct Piece8;
template <> struct Piece8<bf16_t> {
    u32x4 v;
    __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const u32x4*>(p); }
    __device__ __forceinline__ float at(int i) const {
        return i & 1 ? __uint_as_float(v[i >> 1] & 0xffff0000u) : __uint_as_float(v[i >> 1] << 16);
    }
};
template <> struct Piece8<float> {
    f32x4 v[2];
    __device__ __forceinline__ void load(const float* p) {
        v[0] = *reinterpret_cast<const f32x4*>(p);
        v[1] = *reinterpret_cast<const f32x4*>(p + 4);
    }
    __device__ __forceinline__ float at(int i) const { return v[i >> 2][i & 3]; }
};

template <typename TX>
__device__ __forceinline__ float piece_max(const Piece8<TX>& p) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(p.at(i)));
    return m;
}

// What the quotients of a row are made from: 127 x overflows where a is near the type's largest value, so numerator and divisor are
// then 2^-8 of themselves (an x that loses bits by it is 0 of a).
struct Divisor { float a, by, times; };
__device__ __forceinline__ Divisor divisor(float a) {
    const float f = a > 1e36f ? 0x1p-8f : 1.f;
    return {a, a * f, 127.f * f};
}

// 127 x / a for bf16 x and a: 127 x and the product of a with an odd number of up to 8 bits are exact in fp32, a quotient that is
// no half is 2^-16 of itself or more away from one, and the division is correctly rounded.
__device__ __forceinline__ int quantize1(bf16_t, float x, const Divisor& d) { return (int)rintf(d.times * x / d.by); }
// fp32: 127 x is rounded, so a quotient next to a half is computed again in 64 bits, where it is exact to 2^-46 and no quotient
// that is no half is within 2^-34 of one.
__device__ __forceinline__ int quantize1(float, float x, const Divisor& d) {
    const float t = d.times * x / d.by;
    float n = rintf(t);
    if (fabsf(fabsf(t - n) - 0.5f) < 1e-4f) n = (float)rint(127.0 * (double)x / (double)d.a);
    return (int)n;
}

// a = 0: a row of zeros, scale 0.
template <typename TX>
__device__ __forceinline__ uint2 quantize8(const Piece8<TX>& p, const Divisor& d) {
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        w[h] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[h] |= ((uint32_t)quantize1(TX(), p.at(h * 4 + i), d) & 0xffu) << (8 * i);
    }
    return d.a > 0.f ? make_uint2(w[0], w[1]) : make_uint2(0u, 0u);
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}

// One row by kQuantThreads threads: HELD pieces a thread stay in registers (0: the row is read twice).  store(i, q) takes the
// 8 bytes of piece i.  red: 4 floats of LDS, which no thread still reads from the call before.
template <typename TX, int HELD, typename Store>
__device__ __forceinline__ float quantize_row(const TX* __restrict__ x, int pieces, float* red, Store store) {
    const int tid = threadIdx.x;
    constexpr int H = HELD > 0 ? HELD : 1;
    Piece8<TX> held[H];
    float m = 0.f;
    if constexpr (HELD > 0) {
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (i * kQuantThreads + tid < pieces) held[i].load(x + (size_t)(i * kQuantThreads + tid) * 8);
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (i * kQuantThreads + tid < pieces) m = fmaxf(m, piece_max(held[i]));
    } else {
        for (int i = tid; i < pieces; i += kQuantThreads) {
            held[0].load(x + (size_t)i * 8);
            m = fmaxf(m, piece_max(held[0]));
        }
    }
    m = wave_max(m);
    if ((tid & 63) == 0) red[tid >> 6] = m;
    __syncthreads();
    const float a = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const Divisor by = divisor(a);
    if constexpr (HELD > 0) {
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (i * kQuantThreads + tid < pieces) store(i * kQuantThreads + tid, quantize8(held[i], by));
    } else {
        for (int i = tid; i < pieces; i += kQuantThreads) {
            held[0].load(x + (size_t)i * 8);
            store(i, quantize8(held[0], by));
        }
    }
    return a;
}

}  // namespace meteora
