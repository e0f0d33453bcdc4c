// Rows as 8-bit whole numbers with one scale each (device side, shared by quant.hip and sort.hip):
//     a = max_i |x_i|,   q_i = 127 x_i / a rounded to the nearest whole number, halves to the even one,   scale = a / 127.
// A row with an infinity or a NaN is zeros with that scale: a product of it is NaN, and no other row's.
// The rounding is the exact quotient's: x_i = a / 2 is 63.5, and bf16 rows hold such values often (one in about 256 of the elements
// of an octave), so whether a half is seen as one decides a whole step of the result.
#pragma once
#include "common.hpp"

namespace meteora {

constexpr int kQuantThreads = 256;

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

// The larger one, NaN if either is: a row that holds a NaN must not come out as numbers.
__device__ __forceinline__ float top2(float a, float b) { return __builtin_elementwise_maximum(a, b); }

template <typename TX>
__device__ __forceinline__ float piece_max(const Piece8<TX>& p) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = top2(m, fabsf(p.at(i)));
    return m;
}

// A row's maximum a, and up * by = 127 / a: `up` brings rows whose 127 / a no fp32 holds to where it does (exactly: 2^64).
struct Divisor { float a, up, by; };
__device__ __forceinline__ Divisor divisor(float a) {
    const float up = a < 0x1p-100f ? 0x1p64f : 1.f;
    return {a, up, 127.f / (a * up)};   // a = 0, infinity or NaN: quantize8 writes zeros
}

// Bits whose low byte is the whole number next to t, |t| < 128: 1.5 * 2^23 has steps of 1.
__device__ __forceinline__ uint32_t whole_bits(float t) { return __float_as_uint(t + 12582912.f); }

// bf16: x = m 2^e and a = n 2^f of 8-bit m, n make 127 x / a a half exactly or leave it 1 / (254 m) > 2^-16 of itself away from one.
// x * by is within 2^-23 of it, so with 17 bits kept, 2^-17 at most moved (2^-17 + 2^-23 < 2^-16), halves are halves and nothing else is or
// crosses one.
__device__ __forceinline__ uint32_t quantize1(bf16_t, float x, const Divisor& d) {
    const uint32_t t = __float_as_uint(x * d.by);
    return whole_bits(__uint_as_float((t + 0x40u) & 0xffffff80u));
}
// fp32: a quotient whose approximation (within 2^-22 of it, 4e-5) is next to a half is computed again in 64 bits, where it is exact to
// 2^-46 and no quotient that is no half is within 2^-34 of one.
__device__ __forceinline__ uint32_t quantize1(float, float x, const Divisor& d) {
    const float t = x * d.by;
    uint32_t n = whole_bits(t);
    if (fabsf(t - (__uint_as_float(n) - 12582912.f)) > 0.4999f)
        n = whole_bits((float)rint(127.0 * (double)x / ((double)d.a * (double)d.up)));
    return n;
}

template <typename TX>
__device__ __forceinline__ uint2 quantize8(const Piece8<TX>& p, const Divisor& d) {
    uint32_t b[8], w[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = quantize1(TX(), d.up == 1.f ? p.at(i) : p.at(i) * d.up, d);   // uniform over the row
#pragma unroll
    for (int h = 0; h < 2; ++h)   // the low bytes of four
        w[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[h * 4 + 3], b[h * 4 + 2], 0x0c0c0400u),
                                     __builtin_amdgcn_perm(b[h * 4 + 1], b[h * 4], 0x0c0c0400u), 0x05040100u);
    return d.a > 0.f && d.a < INFINITY ? make_uint2(w[0], w[1]) : make_uint2(0u, 0u);
}

// A row by G threads (a wavefront, or the 4 of a workgroup).  HELD pieces a thread stay in registers between the two passes; 0: the row
// is read twice.
template <typename TX, int G, int HELD>
struct QuantRow {
    static constexpr int H = HELD > 0 ? HELD : 1;
    Piece8<TX> held[H];
    __device__ __forceinline__ void load(const TX* __restrict__ x, int pieces) {
        const int lane = threadIdx.x & (G - 1);
        if constexpr (HELD > 0)
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                if (i * G + lane < pieces) held[i].load(x + (size_t)(i * G + lane) * 8);
    }
    // max |x|; red: 4 floats of LDS that no thread still reads (G = 256 only, which waits for all of them)
    __device__ __forceinline__ float top(const TX* __restrict__ x, int pieces, float* red) {
        const int lane = threadIdx.x & (G - 1);
        float m = 0.f;
        if constexpr (HELD > 0) {
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                if (i * G + lane < pieces) m = top2(m, piece_max(held[i]));
        } else {
            for (int i = lane; i < pieces; i += G) {
                held[0].load(x + (size_t)i * 8);
                m = top2(m, piece_max(held[0]));
            }
        }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) m = top2(m, __shfl_xor(m, off));
        if constexpr (G == 64) return m;
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
        __syncthreads();
        return top2(top2(red[0], red[1]), top2(red[2], red[3]));
    }
    // store(i, q) takes the 8 bytes of piece i
    template <typename Store>
    __device__ __forceinline__ void store(const TX* __restrict__ x, int pieces, float a, Store put) {
        const int lane = threadIdx.x & (G - 1);
        const Divisor d = divisor(a);
        if constexpr (HELD > 0) {
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                if (i * G + lane < pieces) put(i * G + lane, quantize8(held[i], d));
        } else {
            for (int i = lane; i < pieces; i += G) {
                held[0].load(x + (size_t)i * 8);
                put(i, quantize8(held[0], d));
            }
        }
    }
};

// The shape of a row of d elements: go(G, HELD) as integral constants.  A wavefront to a row of up to 512 elements, and with `many` rows
// to one of up to 2048; a workgroup to longer ones, and rows of more than 16384 are read twice.  quantize_rows, wavefront and workgroup:
// 16384 x 1024 12.8 and 17.5 us, 4096 x 4096 12.2 and 11.7, 2048 x 8192 13.8 and 11.6.
template <typename F>
static hipError_t quant_row_shape(int d, bool many, F go) {
    using std::integral_constant;
    const int pieces = d / 8;
    if (pieces <= 64) return go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    if (pieces <= 256 && many) return go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    if (pieces <= 256) return go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    if (pieces <= 512) return go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    if (pieces <= 1024) return go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    if (pieces <= 2048) return go(integral_constant<int, 256>{}, integral_constant<int, 8>{});
    return go(integral_constant<int, 256>{}, integral_constant<int, 0>{});
}

}  // namespace meteora
