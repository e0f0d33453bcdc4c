// Rows as 4-bit values with a power of two for every 32 inputs (device side).  With a = max |x_i| over a block of 32 consecutive inputs:
//     E = max(0, floor(log2 a) - 2 + 127),   q_i = the E2M1 value nearest to x_i 2^(127 - E), ties to the even code, at most 6
// so that the block's largest value comes to lie in [4, 8) (above 6 it is 6).  The byte E (E8M0) stands for 2^(E - 127).  A block of zeros, or
// of nothing but values below 2^-125, has E = 0.  A block with an infinity or a NaN is zeros with E = 255, which stands for NaN: products
// of its row are NaN and no other row's.
//
// Two codes a byte, the first one low.  Scales of 16 blocks (512 inputs, a chunk) lie next to each other, those of a chunk's rows behind
// each other: scale[ceil(d / 512)][rows][16], that of block b of row t at [b / 16][t][(b % 4) * 4 + b % 16 / 4], zeros behind the last.
// A matrix instruction over 128 inputs takes the scale of block kq from the lanes of quarter kq: these four bytes, the quarter's scales of
// four instructions, are one word of a lane, and the words of 16 rows are 256 consecutive bytes.
#pragma once
#include "common.hpp"
#include "quant.hpp"

namespace meteora {

constexpr int kMxBlock = 32, kMxChunk = 512;
__host__ __device__ constexpr int mx4_chunks(int d) { return (d + kMxChunk - 1) / kMxChunk; }
__host__ __device__ constexpr size_t mx4_scale_bytes(int rows, int d) { return (size_t)mx4_chunks(d) * (size_t)rows * 16; }

// 2^(E - 127), also where that is no normal number; NaN for 255.
__device__ __forceinline__ float mx4_scale(uint32_t E) {
    return __uint_as_float(E == 0 ? 0x00400000u : E == 255 ? 0x7fc00000u : E << 23);
}

// the greater of two |x| as whole numbers: infinities above all numbers, NaN above those
__device__ __forceinline__ uint32_t top_bits(const Piece8<bf16_t>& p) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t v = p.v[i] & 0x7fff7fffu;
        m = max(m, max(v & 0xffff0000u, v << 16));
    }
    return m;
}
__device__ __forceinline__ uint32_t top_bits(const Piece8<float>& p) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(p.at(i)) & 0x7fffffffu);
    return m;
}
// of the block that the four lanes of a quad hold
template <typename TX>
__device__ __forceinline__ uint32_t mx4_exponent(const Piece8<TX>& p) {
    uint32_t m = top_bits(p);
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xf, 0xf, true));   // quad_perm 1 0 3 2
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xf, 0xf, true));   // quad_perm 2 3 0 1
    const uint32_t e = m >> 23;
    return e == 255 ? 255 : (uint32_t)max((int)e - 2, 0);
}

// v_cvt_scalef32_pk_fp4 divides by a power of two, rounds to the nearest value, ties to the even code, and stays at 6 above.
__device__ __forceinline__ uint32_t mx4_quantize8(const Piece8<bf16_t>& p, uint32_t E) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const float s = mx4_scale(E);
    const uint32_t v0 = p.v[0], v1 = p.v[1], v2 = p.v[2], v3 = p.v[3];
    uint32_t q = 0;
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(bf16x2, v0), s, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(bf16x2, v1), s, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(bf16x2, v2), s, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(bf16x2, v3), s, 3);
    return E == 255 ? 0 : q;
}
__device__ __forceinline__ uint32_t mx4_quantize8(const Piece8<float>& p, uint32_t E) {
    const float s = mx4_scale(E);
    uint32_t q = 0;
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, p.at(0), p.at(1), s, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, p.at(2), p.at(3), s, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, p.at(4), p.at(5), s, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, p.at(6), p.at(7), s, 3);
    return E == 255 ? 0 : q;
}

// 8 codes as bf16 values: exact, but for those that bf16 does not hold (above 2^128; under 2^-133, which no block that was quantised has)
__device__ __forceinline__ u32x4 mx4_bf16x8(uint32_t q, float s) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 3))};
}

// The scales of `rows` consecutive rows of an operand with `all` rows, a chunk at a time.  Rows past the last give 0, which stands for
// 2^-127, and so does a chunk past the last.
struct ScaleRows {
    const uint8_t* first;
    size_t step;          // bytes from chunk to chunk
    int bytes, chunks;
    __device__ __forceinline__ ScaleRows(const uint8_t* scale, int all, int row0, int rows, int row_bytes)
        : first(scale + (size_t)row0 * 16), step((size_t)all * 16), bytes(rows * 16), chunks((row_bytes + 255) / 256) {}
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t chunk(int c) const {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(first + (size_t)c * step), 0, c < chunks ? (uint32_t)bytes : 0u,
                                                 0x00020000);
    }
};

__device__ __forceinline__ void mx4_scale_lds(__amdgpu_buffer_rsrc_t rsrc, unsigned char* dst, uint32_t voff) {   // a word to each lane
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)dst, 4, voff, 0, 0, 0);
}

}  // namespace meteora
