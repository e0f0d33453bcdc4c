// Products of 8-bit whole numbers with a scale per token and per output channel, over groups of consecutive rows:
//
//     out[t,c] = qs[t] * ws[e,c] * sum_i q[t,i] * W_e[c,i],     offsets[e] <= t < offsets[e+1]   (one group: the dense product)
//
// The sum is exact: |q|, |W| <= 128, so 131056 inputs stay below 2^31.  Nothing depends on the order it is taken in, and results
// are the same whichever kernel and tile computes them.  fp32 holds it to 2^-24; two products with the scales, one rounding to
// bf16 where the output is that.
//
// gemm_i8_stream_kernel   any size: a workgroup's wavefronts split K between them and add their tiles in LDS; operands go from
//                         memory to registers in the matrix cores' order.
#include "common.hpp"
#include "kernels.hpp"

namespace meteora {

typedef __attribute__((__vector_size__(4 * sizeof(int32_t)))) int32_t i32x4;

struct GemmI8Args {
    const int8_t* q;        // [T, d_in]
    const float* q_scale;   // [T]
    const int8_t* W;        // [N, d_out, d_in]
    const float* w_scale;   // [N, d_out]
    const int32_t* offsets; // [N+1], or nullptr: one group of all rows
    void* out;              // [T, d_out]
    int T, d_in, d_out, N;
    int tiles_m, tiles_n;   // row tiles of the grid (at least as many as there are), column tiles
};

// Rows [row0, row0 + rows) of group e: row tile `tile` of all groups, each cut into tiles of BM rows.  rows = 0: there is no such
// tile.  Whatever the offsets hold, the rows lie in [0, T).
struct RowTile { int e, row0, rows; };

template <int BM>
__device__ __forceinline__ RowTile row_tile(const GemmI8Args& a, int tile, int lane) {
    if (a.offsets == nullptr) return {0, tile * BM, min(BM, a.T - tile * BM)};
    int lo = 0, hi = 0;
    if (lane < a.N) {
        lo = min(max(a.offsets[lane], 0), a.T);
        hi = min(max(a.offsets[lane + 1], lo), a.T);
    }
    const int mine = (hi - lo + BM - 1) / BM;
    int end = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int n = __shfl_up(end, off);
        if (lane >= off) end += n;
    }
    const unsigned long long after = __ballot(end > tile);
    if (after == 0) return {0, 0, 0};
    const int e = __ffsll(after) - 1;
    const int first = __shfl(lo, e) + (tile - (__shfl(end, e) - __shfl(mine, e))) * BM;
    return {e, first, min(BM, __shfl(hi, e) - first)};
}

// The workgroups of an XCD take consecutive tiles (ids are dealt to the 8 XCDs in turn), row tiles of the same columns of W
// next to each other.
__device__ __forceinline__ int xcd_order(int wg, int total) {
    const int per = total / 8, rest = total % 8, xcd = wg % 8;
    return xcd * per + min(xcd, rest) + wg / 8;
}

constexpr int kStreamWaves = 8;
constexpr uint32_t kOutside = 0x80000000u;   // past every resource here, also with a K offset added

template <int TB, int RB> constexpr int stream_i8_lds() { return kStreamWaves * TB * RB * 1024; }

template <typename TO>
__device__ __forceinline__ void store4(TO* dst, const float (&v)[4]);
template <>
__device__ __forceinline__ void store4<float>(float* dst, const float (&v)[4]) {
    *reinterpret_cast<f32x4*>(dst) = f32x4{v[0], v[1], v[2], v[3]};
}
template <>
__device__ __forceinline__ void store4<bf16_t>(bf16_t* dst, const float (&v)[4]) {
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

// TB x 16 rows of q, RB x 16 rows of W.
template <typename TO, int TB, int RB>
__global__ __launch_bounds__(kStreamWaves * 64) void gemm_i8_stream_kernel(const GemmI8Args a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, kq = lane >> 4;
    const int id = xcd_order(blockIdx.x, a.tiles_m * a.tiles_n);
    const int tile_n = id / a.tiles_m;
    const RowTile rt = row_tile<TB * 16>(a, id - tile_n * a.tiles_m, lane);
    const int rows = __builtin_amdgcn_readfirstlane(rt.rows), e = __builtin_amdgcn_readfirstlane(rt.e);
    const int row0 = __builtin_amdgcn_readfirstlane(rt.row0);
    if (rows <= 0) return;
    const int n0 = tile_n * RB * 16, cols = min(RB * 16, a.d_out - n0);
    const uint32_t ld = (uint32_t)a.d_in;
    const __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(a.q + (size_t)row0 * ld), 0,
                                                                        (uint32_t)rows * ld, 0x00020000);
    const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<int8_t*>(a.W + ((size_t)e * a.d_out + n0) * ld), 0, (uint32_t)cols * ld, 0x00020000);

    i32x4 acc[TB][RB];
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int r = 0; r < RB; ++r) acc[t][r] = i32x4{0, 0, 0, 0};

    // A step is 128 bytes of every row, a wavefront takes every eighth; a lane holds 32 bytes in a row of them, 16 for each of two
    // MFMAs.  Rows past the tile's last load zeros, as do columns past d_in.
    for (uint32_t k0 = (uint32_t)wave * 128; k0 < ld; k0 += kStreamWaves * 128) {
        u32x4 x[2][TB], w[2][RB];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t k = k0 + (uint32_t)(kq * 32 + h * 16);
#pragma unroll
            for (int r = 0; r < RB; ++r)
                w[h][r] = __builtin_amdgcn_raw_buffer_load_b128(wr, k < ld ? (uint32_t)(r * 16 + l15) * ld + k : kOutside, 0, 0);
#pragma unroll
            for (int t = 0; t < TB; ++t)
                x[h][t] = __builtin_amdgcn_raw_buffer_load_b128(xr, k < ld ? (uint32_t)(t * 16 + l15) * ld + k : kOutside, 0, 0);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < TB; ++t)
#pragma unroll
                for (int r = 0; r < RB; ++r)
                    acc[t][r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, w[h][r]),
                                                                      __builtin_bit_cast(i32x4, x[h][t]), acc[t][r], 0, 0, 0);
    }

    // W is the first operand: a lane holds 4 consecutive columns of row l15 of a block.  [wave][block][lane] in LDS.
    i32x4* part = reinterpret_cast<i32x4*>(smem);
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int r = 0; r < RB; ++r) part[(wave * TB * RB + t * RB + r) * 64 + lane] = acc[t][r];
    __syncthreads();
    for (int b = wave; b < TB * RB; b += kStreamWaves) {
        const int t = b / RB, r = b % RB;
        const int row = t * 16 + l15, col = r * 16 + kq * 4;   // d_out % 8 == 0: 4 columns are all in or all out
        if (row >= rows || col >= cols) continue;
        i32x4 sum = part[b * 64 + lane];
#pragma unroll
        for (int v = 1; v < kStreamWaves; ++v) sum += part[(v * TB * RB + b) * 64 + lane];
        const float qs = a.q_scale[row0 + row];
        const f32x4 ws = *reinterpret_cast<const f32x4*>(a.w_scale + (size_t)e * a.d_out + n0 + col);
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)sum[i] * qs * ws[i];
        store4((TO*)a.out + (size_t)(row0 + row) * a.d_out + n0 + col, v);
    }
}

template <typename TO, int TB, int RB>
static hipError_t launch_stream(GemmI8Args a, hipStream_t stream) {
    a.tiles_m = ceil_div(a.T, TB * 16) + (a.offsets != nullptr ? a.N - 1 : 0);   // every group may end in a partial tile
    a.tiles_n = ceil_div(a.d_out, RB * 16);
    constexpr int lds = stream_i8_lds<TB, RB>();
    const auto kern = &gemm_i8_stream_kernel<TO, TB, RB>;
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(kern), lds);
    if (e != hipSuccess) return e;
    if ((int64_t)a.tiles_m * a.tiles_n >= INT32_MAX) return hipErrorInvalidValue;
    kern<<<a.tiles_m * a.tiles_n, kStreamWaves * 64, lds, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_gemm_i8(const int8_t* q, const float* q_scale, const int8_t* W, const float* w_scale, const int32_t* offsets,
                          int T, int d_in, int d_out, int N, bool bf16, void* out, hipStream_t stream) {
    GemmI8Args a{q, q_scale, W, w_scale, offsets, out, T, d_in, d_out, N, 0, 0};
    return bf16 ? launch_stream<bf16_t, 4, 2>(a, stream) : launch_stream<float, 4, 2>(a, stream);
}

hipError_t gemm_i8_init_kernels() {
    hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(&gemm_i8_stream_kernel<bf16_t, 4, 2>), stream_i8_lds<4, 2>());
    if (e == hipSuccess)
        e = ensure_lds_limit(reinterpret_cast<const void*>(&gemm_i8_stream_kernel<float, 4, 2>), stream_i8_lds<4, 2>());
    return e;
}

}  // namespace meteora
