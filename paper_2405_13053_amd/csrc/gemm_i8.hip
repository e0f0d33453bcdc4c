// Products of 8-bit whole numbers with a scale per token and per output channel, over groups of consecutive rows:
//
//     out[t,c] = qs[t] * ws[e,c] * sum_i q[t,i] * W_e[c,i],     offsets[e] <= t < offsets[e+1]   (one group: the dense product)
//
// The sum is exact: |q|, |W| <= 128, so 131056 inputs stay below 2^31.  Nothing depends on the order it is taken in, and results
// are the same whichever kernel and tile computes them.  fp32 holds it to 2^-24; two products with the scales, one rounding to
// bf16 where the output is that.
//
// gemm_i8_ring_kernel   many rows: output tiles of 64 x 64 to 256 x 256, operands through rings of LDS slots
// gemm_i8_wave_kernel   few rows: a workgroup's wavefronts split K between them, each with a ring of its own, and add their tiles in LDS
// gemm_i8_one_kernel    up to 128 inputs: the output is what there is to move
// gemm_i8_row_kernel    up to 4 tokens of meteora_base_gemm_i8: their quantisation too
#include "common.hpp"
#include "gemm_mfma.hpp"
#include "gemm_rows.hpp"
#include "kernels.hpp"
#include "quant.hpp"

namespace meteora {

typedef __attribute__((__vector_size__(4 * sizeof(int32_t)))) int32_t i32x4;

using GemmI8Args = GemmRowsArgs<float>;   // q_scale[T], w_scale[N, d_out]

template <int TB, int RB, int WV, int D>
constexpr int wave_i8_lds() {
    constexpr int ring = WV * D * (TB + RB) * 2048, sums = WV * TB * RB * 1024;
    return ring > sums ? ring : sums;
}

// The wavefronts' tiles are added in LDS ([wave][block][lane]) and leave as scaled rows.  W is the first operand, so a lane holds 4
// consecutive columns of row l15 of a block; qs, ws: the scales of the blocks wave, wave + WV, ...
template <typename TO, int TB, int RB, int WV, int OUT>
__device__ __forceinline__ void wave_i8_sums(const GemmI8Args& a, const i32x4 (&acc)[TB][RB], unsigned char* smem, const float (&qs)[OUT],
                                             const f32x4 (&ws)[OUT], int row0, int rows, int n0, int cols, int wave, int lane) {
    const int l15 = lane & 15, kq = lane >> 4;
    i32x4* part = reinterpret_cast<i32x4*>(smem);
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int r = 0; r < RB; ++r) part[(wave * TB * RB + t * RB + r) * 64 + lane] = acc[t][r];
    __syncthreads();
#pragma unroll
    for (int u = 0; u < OUT; ++u) {
        const int b = wave + u * WV;
        const int row = b / RB * 16 + l15, col = b % RB * 16 + kq * 4;   // d_out % 8 == 0: 4 columns are all in or all out
        if (b >= TB * RB || row >= rows || col >= cols) continue;
        i32x4 sum = part[b * 64 + lane];
#pragma unroll
        for (int v = 1; v < WV; ++v) sum += part[(v * TB * RB + b) * 64 + lane];
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)sum[i] * qs[u] * ws[u][i];
        store4((TO*)a.out + (size_t)(row0 + row) * a.d_out + n0 + col, v);
    }
}

// Few rows: TB x 16 rows of q, RB x 16 rows of W, WV wavefronts, each with every WV-th K tile of 128 inputs and a ring of its own of
// D slots, so that no wavefront waits for another before the end.
template <typename TO, int TB, int RB, int WV, int D>
__global__ __launch_bounds__(WV * 64) void gemm_i8_wave_kernel(const GemmI8Args a) {
    constexpr int NX = 2 * TB, NW = 2 * RB, NL = NX + NW;   // load instructions per K tile, 8 rows each
    constexpr int NM = 2 * TB * RB;                         // MFMAs per K tile
    static_assert(D >= 2 && (D - 2) * NL < 64, "vmcnt");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, kq = lane >> 4;
    const RowTiles<TB * 16> row_tiles(a, lane);
    if ((int)blockIdx.x >= row_tiles.count * a.tiles_n) return;
    const int id = xcd_order(blockIdx.x, row_tiles.count * a.tiles_n);
    const int tile_n = id / row_tiles.count;
    const RowTile rt = row_tiles.at(a, id - tile_n * row_tiles.count);
    const int rows = rt.rows, e = rt.e, row0 = rt.row0;
    const int n0 = tile_n * a.tile_cols, cols = min(a.tile_cols, a.d_out - n0);
    const uint32_t ld = (uint32_t)a.d_in;
    unsigned char* const ring = smem + wave * D * (TB + RB) * 2048;

    // scales of the blocks that this wavefront writes in the end: on their way before anything else
    constexpr int OUT = (TB * RB + WV - 1) / WV;
    float qs[OUT];
    f32x4 ws[OUT];
#pragma unroll
    for (int u = 0; u < OUT; ++u) {
        const int b = min(wave + u * WV, TB * RB - 1);
        qs[u] = a.q_scale[row0 + min(b / RB * 16 + l15, rows - 1)];
        ws[u] = *reinterpret_cast<const f32x4*>(a.w_scale + (size_t)e * a.d_out + n0 + min(b % RB * 16 + kq * 4, cols - 4));
    }

    WaveOperand<TB> x(a.q + (size_t)row0 * ld, rows, ld, lane);
    WaveOperand<RB> w(a.W + ((size_t)e * a.d_out + n0) * ld, cols, ld, lane);
    const int nk = ceil_div(a.d_in, 128), n = wave < nk ? (nk - 1 - wave) / WV + 1 : 0;
    auto at_tile = [&](int kt) {
        x.at_tile(kt, nk);
        w.at_tile(kt, nk);
    };
    auto request = [&](unsigned char* slot, int i) {   // load i of that K tile: W's first
        if (i < NW) w.template request<kReadOnceI8>(slot, i);
        else x.template request<0>(slot + NW * 1024, i - NW);
    };
#pragma unroll
    for (int d = 0; d < D; ++d) {
        at_tile(wave + d * WV);
#pragma unroll
        for (int i = 0; i < NL; ++i) request(ring + d * (TB + RB) * 2048, i);
    }
    i32x4 acc[TB][RB];
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int r = 0; r < RB; ++r) acc[t][r] = i32x4{0, 0, 0, 0};
    struct Frag { u32x4 x[2][TB], w[2][RB]; };
    auto read = [&](Frag& f, const unsigned char* slot) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const int at = l15 * 128 + swz(l15, ks * 4 + kq) * 16;   // row l15 of a block of 16
#pragma unroll
            for (int r = 0; r < RB; ++r) f.w[ks][r] = *reinterpret_cast<const u32x4*>(slot + r * 2048 + at);
#pragma unroll
            for (int t = 0; t < TB; ++t) f.x[ks][t] = *reinterpret_cast<const u32x4*>(slot + (RB + t) * 2048 + at);
        }
    };
    int slot = 0, kt = wave + D * WV;   // of the tile that is multiplied; the one that is requested
    // multiplies `cur` while `nxt` is read and the tile D ahead is requested into the slot that cur came from
    auto step = [&](Frag& cur, Frag& nxt) {
        unsigned char* const mine = ring + slot * (TB + RB) * 2048;
        slot = slot + 1 == D ? 0 : slot + 1;
        // the next tile has landed: of the loads only those of the D - 2 tiles behind it may be in flight; cur has left its slot
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((D - 2) * NL) : "memory");
        read(nxt, ring + slot * (TB + RB) * 2048);
        at_tile(kt);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            request(mine, i);
#pragma unroll
            for (int m = i * NM / NL; m < (i + 1) * NM / NL; ++m) {
                const int ks = m / (TB * RB), t = m / RB % TB, r = m % RB;
                acc[t][r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, cur.w[ks][r]),
                                                                  __builtin_bit_cast(i32x4, cur.x[ks][t]), acc[t][r], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        kt += WV;
    };
    Frag f0, f1;
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * NL < 64 ? (D - 1) * NL : 63) : "memory");
    read(f0, ring);
    int i = 0;
    for (; i + 1 < n; i += 2) {
        step(f0, f1);
        step(f1, f0);
    }
    if (i < n) step(f0, f1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may land in what follows
    __syncthreads();

    wave_i8_sums<TO, TB, RB, WV>(a, acc, smem, qs, ws, row0, rows, n0, cols, wave, lane);
}

// ------------------------------------------------------------------------------------------
// A few tokens and their quantisation in one launch (meteora_base_gemm_i8): every workgroup quantises all of x itself, into LDS, while
// the first tiles of W are on their way.  That reads x once per workgroup from L2, which up to 32 KB of it (bf16) costs less than the launch.
// W goes through the wavefronts' rings as above; a lane without a row of its own multiplies another's, and its result is not kept.
// ------------------------------------------------------------------------------------------
constexpr int kRowThreads = 256, kRowMaxTokens = 4, kRowMaxBytes = 16384;   // T * d_in, x in 8 bits
constexpr int row_i8_stride(int d_in) { return (d_in + 127) / 128 * 128 + 16; }   // rows start 4 banks apart
template <int RB, int D>
constexpr int row_i8_ring_bytes() { return 4 * D * RB * 2048; }   // and the sums in its place
template <int RB, int D>
constexpr int row_i8_lds_most() { return row_i8_ring_bytes<RB, D>() + kRowMaxBytes + kRowMaxTokens * (127 + 16); }

template <typename TX, int RB, int D, int G, int HELD>
__global__ __launch_bounds__(kRowThreads) void gemm_i8_row_kernel(const GemmI8Args a, const TX* __restrict__ x) {
    constexpr int WV = 4, NL = 2 * RB;
    static_assert(kRowThreads == kQuantThreads && D >= 2 && (D - 1) * NL < 64, "a workgroup quantises a row; vmcnt");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ float red[4], row_scale[kRowMaxTokens];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, kq = lane >> 4;
    const int n0 = xcd_order(blockIdx.x, a.tiles_n) * a.tile_cols, cols = min(a.tile_cols, a.d_out - n0);
    const uint32_t ld = (uint32_t)a.d_in;
    unsigned char* const ring = smem + wave * D * RB * 2048;
    unsigned char* const xq = smem + row_i8_ring_bytes<RB, D>();
    const int stride = row_i8_stride(a.d_in);

    WaveOperand<RB> w(a.W + (size_t)n0 * ld, cols, ld, lane);
    const int nk = ceil_div(a.d_in, 128), n = wave < nk ? (nk - 1 - wave) / WV + 1 : 0;
#pragma unroll
    for (int d = 0; d < D; ++d) {
        w.at_tile(wave + d * WV, nk);
#pragma unroll
        for (int i = 0; i < NL; ++i) w.template request<kReadOnceI8>(ring + d * RB * 2048, i);
    }
    {
        // one row by the workgroup, several by a wavefront each
        QuantRow<TX, G, HELD> r;
        const int pieces = a.d_in / 8;
        for (int t = tid / G; t < a.T; t += kRowThreads / G) {
            const TX* src = x + (size_t)t * a.d_in;
            r.load(src, pieces);
            const float top = r.top(src, pieces, red);
            r.store(src, pieces, top, [&](int i, uint2 v) { *reinterpret_cast<uint2*>(xq + t * stride + i * 8) = v; });
            if ((tid & (G - 1)) == 0) row_scale[t] = top / 127.f;
        }
    }
    float qs[(RB + WV - 1) / WV];
    f32x4 ws[(RB + WV - 1) / WV];
    constexpr int OUT = (RB + WV - 1) / WV;
#pragma unroll
    for (int u = 0; u < OUT; ++u) {
        const int b = min(wave + u * WV, RB - 1);
        ws[u] = *reinterpret_cast<const f32x4*>(a.w_scale + n0 + min(b * 16 + kq * 4, cols - 4));
    }
    __syncthreads();   // x is there (and so are W's first tiles: the compiler has waited for the loads of x, which are younger)
#pragma unroll
    for (int u = 0; u < OUT; ++u) qs[u] = row_scale[min(l15, a.T - 1)];
    const unsigned char* const mine = xq + (l15 % a.T) * stride;

    i32x4 acc[1][RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) acc[0][r] = i32x4{0, 0, 0, 0};
    int slot = 0;
    for (int i = 0; i < n; ++i) {
        // of the loads only those of the D - 1 tiles behind this one may be in flight
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * NL) : "memory");
        u32x4 wf[2][RB], xf[2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
            for (int r = 0; r < RB; ++r)
                wf[ks][r] = *reinterpret_cast<const u32x4*>(ring + (slot * RB + r) * 2048 + l15 * 128 + swz(l15, ks * 4 + kq) * 16);
            xf[ks] = *reinterpret_cast<const u32x4*>(mine + (wave + i * WV) * 128 + (ks * 4 + kq) * 16);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slot is read
        w.at_tile(wave + (i + D) * WV, nk);
#pragma unroll
        for (int j = 0; j < NL; ++j) w.template request<kReadOnceI8>(ring + slot * RB * 2048, j);
        slot = slot + 1 == D ? 0 : slot + 1;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int r = 0; r < RB; ++r)
                acc[0][r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, wf[ks][r]),
                                                                  __builtin_bit_cast(i32x4, xf[ks]), acc[0][r], 0, 0, 0);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may land in what follows
    __syncthreads();
    wave_i8_sums<TX, 1, RB, WV>(a, acc, smem, qs, ws, 0, a.T, n0, cols, wave, lane);
}

// ------------------------------------------------------------------------------------------
// Many rows.  A K tile of 128 inputs is 128 bytes a row, a matrix instruction 16x16x64 takes 16 bytes a lane and as many cycles as
// 16x16x32 does in bf16: byte for byte and cycle for cycle this is the schedule of gemm_mfma_ring_kernel (rings of D slots for the
// rows and D + 1 for W, one barrier per K tile, the next tiles' loads spread over the MFMAs), with whole numbers in the accumulators.
// As there the instruction is written in assembly with its accumulator tied, and the same care is due: the source states the order of
// MFMAs, LDS reads and loads, only MFMAs touch an accumulator inside the K loop, wait states stand in front of the first and behind
// the last (tests/test_mfma_waits_i8_host.py reads the assembly).
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ void mfma16_i8(i32x4& acc, const bf16x8& w, const bf16x8& x) {   // 16 bytes of each
    asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(acc) : "v"(w), "v"(x));
}

template <int MB, int NB, int D>
constexpr int ring_i8_lds() {
    constexpr int ring = (D * MB + (D + 1) * NB) * 32 * kI8Tile, stage = 4 * 32 * (NB * 64 + 16);
    return ring > stage ? ring : stage;
}

// The tile leaves by way of LDS, 32 (16) rows a wavefront at a time, so that stores are 16-byte pieces of whole rows.  Through the L2,
// see kWriteThrough.
template <typename TO, int MB, int NB>
__device__ __forceinline__ void ring_i8_epilogue(const GemmI8Args& a, i32x4 (&acc)[MB][NB], unsigned char* smem, int e, int row0,
                                                 int rows, int n0, int wm, int wn, int wave, int lane) {
    constexpr int EB = sizeof(TO), RS = MB % 2 == 0 ? 32 : 16;
    constexpr int EST = NB * 16 * EB + 16, PPR = NB * EB, NP = RS * PPR / 64;   // bytes and pieces per staged row, pieces per lane
    static_assert(RS * PPR % 64 == 0, "whole wavefronts of pieces");
    const int l15 = lane & 15, kq = lane >> 4;
    float qs[MB];
    f32x4 ws[NB];
    const float* w_scale = a.w_scale + (size_t)e * a.d_out;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) qs[mb] = a.q_scale[row0 + min(wm + mb * 16 + l15, rows - 1)];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)   // d_out % 8 == 0: 4 columns are all in or all out
        ws[nb] = *reinterpret_cast<const f32x4*>(w_scale + min(n0 + wn + nb * 16 + kq * 4, a.d_out - 4));
    __syncthreads();   // every wavefront is done with the operand tiles
    unsigned char* ep = smem + wave * RS * EST;
    const uint32_t row_bytes = (uint32_t)a.d_out * EB;
    const __amdgpu_buffer_rsrc_t out = __builtin_amdgcn_make_buffer_rsrc((TO*)a.out + (size_t)row0 * a.d_out, 0,
                                                                         (uint32_t)rows * row_bytes, 0x00020000);
    auto sync = [] {   // orders this wavefront's own LDS accesses
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
#pragma unroll
    for (int mb = 0; mb < MB; mb += RS / 16) {
#pragma unroll
        for (int h = 0; h < RS / 16; ++h)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = (float)acc[mb + h][nb][i] * qs[mb + h] * ws[nb][i];
                store4(reinterpret_cast<TO*>(ep + (h * 16 + l15) * EST + (nb * 16 + kq * 4) * EB), v);
            }
        sync();
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int p = i * 64 + lane, r = p / PPR, c = p % PPR;
            const int col = n0 + wn + c * (16 / EB);
            const u32x4 v = *reinterpret_cast<const u32x4*>(ep + r * EST + c * 16);
            // rows past the tile's last are past the resource's end, and so are the pieces sent there for their column
            const uint32_t at = col < a.d_out ? (uint32_t)(wm + mb * 16 + r) * row_bytes + (uint32_t)col * EB : 0xffffffffu;
            __builtin_amdgcn_raw_buffer_store_b128(v, out, at, 0, kWriteThrough);
        }
        sync();
        __builtin_amdgcn_sched_barrier(0);   // accumulators leave their registers 32 rows at a time
    }
}

// One tile.  PART: d_in may end in a partial K tile.  ONCE: no other workgroup reads these rows of W.
template <typename TO, int MB, int NB, int D, bool PART, bool ONCE>
__device__ __forceinline__ void ring_i8_tile(const GemmI8Args& a, unsigned char* smem, int e, int row0, int rows, int n0) {
    constexpr int BM = MB * 32, BN = NB * 32, PX = MB, PW = NB;   // 2 x 2 wavefronts; load instructions per wavefront and tile
    static_assert((NB % 2 == 0 || MB % 2 == 0) && D >= 2 && D <= 5 && (D - 1) * (PX + PW) < 64, "2 x 2 micro-blocks; vmcnt");
    constexpr int NR = MB + NB, NM = MB * NB;   // fragment reads and MFMAs per k-step of 64
    constexpr int RA = NM * 3 / 4 / NR > 0 ? NM * 3 / 4 / NR : 1, RB = NM / NR;   // MFMAs per read, see the bf16 kernel
    static_assert(RB >= 1, "a k-step needs one MFMA per fragment read");
    bf16_t* ring = reinterpret_cast<bf16_t*>(smem);
    constexpr int kXElems = BM * kGemmBK, kWElems = BN * kGemmBK;   // in units of two bytes, as everything that is shared

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
    const int l15 = lane & 15, kq = lane >> 4, cols = min(BN, a.d_out - n0);

    const int nk_main = a.d_in / kI8Tile, nk = nk_main + (PART && a.d_in % kI8Tile != 0 ? 1 : 0);
    const int8_t* xb = a.q + (size_t)row0 * a.d_in;
    const int8_t* wb = a.W + ((size_t)e * a.d_out + n0) * a.d_in;
    const DmaOperand ox = dma_operand(reinterpret_cast<const bf16_t*>(xb), rows, a.d_in / 2, 0, wave, lane);
    const DmaOperand ow = dma_operand(reinterpret_cast<const bf16_t*>(wb), cols, a.d_in / 2, 0, wave, lane);
    const PartTile part = part_tile(a.d_in / 2, wave, lane);
    const uint32_t x_bytes = (uint32_t)rows * (uint32_t)a.d_in, w_bytes = (uint32_t)cols * (uint32_t)a.d_in;

    auto xslot = [&](int it) { return ring + (it % D) * kXElems; };
    auto wslot = [&](int it) { return ring + D * kXElems + (it % (D + 1)) * kWElems; };
    auto request_x = [&](bf16_t* slot, int kt, int i, auto is_part) {
        if constexpr (decltype(is_part)::value) dma_piece_behind<true, false>(slot, ox, x_bytes, ox, part, -1, i, wave);
        else dma_piece(slot, ox, kt, i, wave);
    };
    auto request_w = [&](bf16_t* slot, int kt, int i, auto is_part) {
        if constexpr (decltype(is_part)::value) dma_piece_behind<true, false>(slot, ow, w_bytes, ow, part, -1, i, wave);
        else dma_piece<ONCE ? kReadOnceI8 : 0>(slot, ow, kt, i, wave);
    };
    auto request_tile = [&](int it, auto is_part) {
#pragma unroll
        for (int i = 0; i < PX; ++i) request_x(xslot(it), it, i, is_part);
#pragma unroll
        for (int i = 0; i < PW; ++i) request_w(wslot(it), it, i, is_part);
    };
#pragma unroll
    for (int t = 0; t < D; ++t)
        if (t < nk_main) request_tile(t, std::false_type{});
    if (PART && nk_main < D && nk > nk_main) request_tile(nk_main, std::true_type{});
    i32x4 acc[MB][NB];   // first values while the first tile is on its way; two wait states or more before the first MFMA
#pragma unroll
    for (int mi = 0; mi < MB; ++mi)
#pragma unroll
        for (int ni = 0; ni < NB; ++ni) {
            acc[mi][ni] = i32x4{0, 0, 0, 0};
            asm volatile("" : "+a"(acc[mi][ni]));
        }
    asm volatile("s_nop 1" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);

    Frags16<MB, NB> f0, f1;
    auto wait_tiles = [&](int left) {   // the loads of at most `left` tiles may still be in flight
        if (D > 4 && left >= 4) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(D > 4 ? 4 * (PX + PW) : 0) : "memory");
        else if (D > 3 && left == 3) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(D > 3 ? 3 * (PX + PW) : 0) : "memory");
        else if (D > 2 && left == 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(D > 2 ? 2 * (PX + PW) : 0) : "memory");
        else if (left == 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(PX + PW) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    wait_tiles(min(nk, D) - 1);   // d_in >= 16: one K tile at least
#pragma unroll
    for (int i = 0; i < NR; ++i) load_frag16<MB, NB>(f0, xslot(0), wslot(0), wm, wn, l15, kq, 0, i);

    auto mfmas = [&](const Frags16<MB, NB>& f, int k0, int k1) {
#pragma unroll
        for (int k = k0; k < k1; ++k)
            mfma16_i8(acc[order_mi<MB, NB>(k)][order_ni<MB, NB>(k)], f.w[order_ni<MB, NB>(k)], f.x[order_mi<MB, NB>(k)]);
    };
    int slot_x = 0, slot_w = D * kXElems;   // where tile `it` lies, outside the unrolled main loop
    // REQ: 0 = tile it + D is a whole one, 1 = it is the partial one, 2 = there is none
    auto tile_step = [&](int it, auto req, auto ph) __attribute__((always_inline)) {
        constexpr int REQ = decltype(req)::value, PH = decltype(ph)::value;
        using IsPart = std::integral_constant<bool, REQ == 1>;
        auto xsl = [&](int d) {   // slots of tile it + d, d = 0, 1 or D
            if constexpr (PH >= 0) return ring + ((PH + d) % D) * kXElems;
            else return ring + (d != 1 ? slot_x : slot_x == (D - 1) * kXElems ? 0 : slot_x + kXElems);
        };
        auto wsl = [&](int d) {
            constexpr int first = D * kXElems, last = first + D * kWElems;
            if constexpr (PH >= 0) return ring + first + ((PH + d) % (D + 1)) * kWElems;
            else if (d == 0) return ring + slot_w;
            else if (d == 1) return ring + (slot_w == last ? first : slot_w + kWElems);
            else return ring + (slot_w == first ? last : slot_w - kWElems);
        };
        const bf16_t* xs = xsl(0);
        const bf16_t* ws = wsl(0);
        bf16_t* const xreq = xsl(D);
        bf16_t* const wreq = wsl(D);
        // k-step 0: its MFMAs, the fragment reads of k-step 1 and the W pieces of tile it + D
        int issued = 0;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            mfmas(f0, i * RA, (i + 1) * RA);
            load_frag16<MB, NB>(f1, xs, ws, wm, wn, l15, kq, 1, i);
            if constexpr (REQ < 2) {
#pragma unroll
                for (int c = 0; c < pieces_after_read(i, PW, NR); ++c) request_w(wreq, it + D, issued++, IsPart{});
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        mfmas(f0, NR * RA, NM);
        __builtin_amdgcn_sched_barrier(0);
        // tile it + 1 must have landed, and every wavefront's reads of tile it must be complete
        if constexpr (REQ < 2)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(PW + (D - 2) * (PX + PW)) : "memory");
        else
            wait_tiles(nk - 2 - it);
        // k-step 1: its MFMAs, the first fragments of tile it + 1 and the row pieces of tile it + D into the slot just drained
        const bf16_t* xn = xsl(1);
        const bf16_t* wnx = wsl(1);
        if constexpr (REQ < 2) {
            issued = 0;
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                mfmas(f1, i * RB, (i + 1) * RB);
                load_frag16<MB, NB>(f0, xn, wnx, wm, wn, l15, kq, 0, i);
#pragma unroll
                for (int c = 0; c < pieces_after_read(i, PX, NR); ++c) request_x(xreq, it + D, issued++, IsPart{});
                __builtin_amdgcn_sched_barrier(0);
            }
            mfmas(f1, NR * RB, NM);
        } else {
            if (it + 1 < nk) {   // reads only: MFMAs in both arms of a branch make the compiler copy accumulators
#pragma unroll
                for (int i = 0; i < NR; ++i) load_frag16<MB, NB>(f0, xn, wnx, wm, wn, l15, kq, 0, i);
            }
            __builtin_amdgcn_sched_barrier(0);
            mfmas(f1, 0, NM);
        }
        if constexpr (PH < 0) {
            slot_x = (int)(xn - ring);
            slot_w = (int)(wnx - ring);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    using Req0 = std::integral_constant<int, 0>;
    using Rt = std::integral_constant<int, -1>;
    int it = 0;
    constexpr int TRIP = D * (D + 1);   // a whole period of both rings: no slot arithmetic between two tiles
    if constexpr (MB >= 6 && D <= 3) {
        for (; it + TRIP - 1 + D < nk_main; it += TRIP)
            for_each_phase(std::make_integer_sequence<int, TRIP>{}, [&](auto ph) __attribute__((always_inline)) {
                tile_step(it + decltype(ph)::value, Req0{}, ph);
            });
        slot_x = (int)(xslot(it) - ring);
        slot_w = (int)(wslot(it) - ring);
    }
    for (; it + D < nk_main; ++it) tile_step(it, Req0{}, Rt{});
    if constexpr (PART)
        for (; it + D < nk; ++it) tile_step(it, std::integral_constant<int, 1>{}, Rt{});
    for (; it < nk; ++it) tile_step(it, std::integral_constant<int, 2>{}, Rt{});
    mfma_drain();
#pragma unroll
    for (int mi = 0; mi < MB; ++mi)
#pragma unroll
        for (int ni = 0; ni < NB; ++ni) asm volatile("" : "+a"(acc[mi][ni]));   // values from here on, not before
    __builtin_amdgcn_sched_barrier(0);
    ring_i8_epilogue<TO, MB, NB>(a, acc, smem, e, row0, rows, n0, wm, wn, wave, lane);
}

// W of a group with one row tile is read once, and where it comes from memory it is requested as such: 8 groups of 4096 -> 4096, 16 and 64 rows
// each, 128 x 128 tiles 32.9 and 33.5 us against 35.7 and 35.6.  Where other row tiles read it again that policy costs 5 to 30%, and where it
// is still in a cache too (28 groups of 4096 -> 64, 7 MB: 12.8 against 11.0).  So the workgroup chooses between two copies of the loop;
// 256 x 256 tiles, which few rows do not come to, have one.
template <typename TO, int MB, int NB, int D, bool PART>
__global__ __launch_bounds__(256) void gemm_i8_ring_kernel(const GemmI8Args a) {
    constexpr int BM = MB * 32, BN = NB * 32;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const RowTiles<BM> row_tiles(a, (int)threadIdx.x & 63);
    const int tiles = row_tiles.count * a.tiles_n;
    if ((int)blockIdx.x >= (a.tail ? tail_start(tiles) : tiles)) return;
    int tile_m, tile_n;
    tile_of_workgroup(blockIdx.x, row_tiles.count, a.tiles_n, tile_m, tile_n);
    const RowTile rt = row_tiles.at(a, tile_m);
    if constexpr (MB * NB < 64)
        if (rt.alone && a.past_caches) {
            ring_i8_tile<TO, MB, NB, D, PART, true>(a, smem, rt.e, rt.row0, rt.rows, tile_n * BN);
            return;
        }
    ring_i8_tile<TO, MB, NB, D, PART, false>(a, smem, rt.e, rt.row0, rt.rows, tile_n * BN);
}

// The 256 x 256 tiles behind tail_start, in smaller ones: as small as one to a CU allows, or two of the largest.  The number of tiles of
// groups is known here only, and so is their size.
template <typename TO, int MB, int NB, int D, bool PART>
__device__ __forceinline__ void tail_i8_part(const GemmI8Args& a, const RowTiles<256>& row_tiles, unsigned char* smem, int first, int tiles) {
    constexpr int BM = MB * 32, BN = NB * 32, PM = 256 / BM, PN = 256 / BN;
    const int id = first + (int)blockIdx.x / (PM * PN), m0 = (int)blockIdx.x % PM * BM;
    if (id >= tiles) return;
    int tile_m, tile_n;
    tile_of_workgroup(id, row_tiles.count, a.tiles_n, tile_m, tile_n);
    const RowTile rt = row_tiles.at(a, tile_m);
    const int rows = min(BM, rt.rows - m0), n0 = tile_n * 256 + (int)blockIdx.x / PM % PN * BN;
    if (rows <= 0 || n0 >= a.d_out) return;
    ring_i8_tile<TO, MB, NB, D, PART, false>(a, smem, rt.e, rt.row0 + m0, rows, n0);
}
constexpr int tail_i8_lds() {   // two workgroups to a CU
    const int a = ring_i8_lds<2, 2, 4>(), b = ring_i8_lds<4, 2, 3>(), c = ring_i8_lds<4, 4, 2>();
    return a > b ? (a > c ? a : c) : (b > c ? b : c);
}
static_assert(2 * tail_i8_lds() <= 160 * 1024, "LDS");

template <typename TO, bool PART>
__global__ __launch_bounds__(256) void gemm_i8_tail_kernel(const GemmI8Args a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const RowTiles<256> row_tiles(a, (int)threadIdx.x & 63);
    const int tiles = row_tiles.count * a.tiles_n, first = tail_start(tiles);
    if (tiles - first <= kTailSmall) tail_i8_part<TO, 2, 2, 4, PART>(a, row_tiles, smem, first, tiles);
    else if (tiles - first <= kTailMiddle) tail_i8_part<TO, 4, 2, 3, PART>(a, row_tiles, smem, first, tiles);
    else tail_i8_part<TO, 4, 4, 2, PART>(a, row_tiles, smem, first, tiles);
}

// Up to 128 inputs (the expand of adapters): one K tile, and the output is what there is to move.  The same tiles without a ring, so
// that four or five workgroups share a CU and one's loads and arithmetic lie under another's stores.
template <typename TO, int MB, int NB>
constexpr int one_i8_lds() {
    constexpr int tiles = (MB + NB) * 32 * kI8Tile, stage = 4 * (MB % 2 == 0 ? 32 : 16) * (NB * 16 * (int)sizeof(TO) + 16);
    return tiles > stage ? tiles : stage;
}

template <typename TO, int MB, int NB>
__global__ __launch_bounds__(256) void gemm_i8_one_kernel(const GemmI8Args a) {
    constexpr int BM = MB * 32, BN = NB * 32;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    bf16_t* xs = reinterpret_cast<bf16_t*>(smem);
    bf16_t* wsm = xs + BM * kGemmBK;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
    const int l15 = lane & 15, kq = lane >> 4;
    const RowTiles<BM> row_tiles(a, lane);
    if ((int)blockIdx.x >= row_tiles.count * a.tiles_n) return;
    int tile_m, tile_n;
    tile_of_workgroup(blockIdx.x, row_tiles.count, a.tiles_n, tile_m, tile_n);
    const RowTile rt = row_tiles.at(a, tile_m);
    const int rows = rt.rows, e = rt.e, row0 = rt.row0;
    const int n0 = tile_n * BN, cols = min(BN, a.d_out - n0);
    const int8_t* xb = a.q + (size_t)row0 * a.d_in;
    const int8_t* wb = a.W + ((size_t)e * a.d_out + n0) * a.d_in;
    const DmaOperand ox = dma_operand(reinterpret_cast<const bf16_t*>(xb), rows, a.d_in / 2, 0, wave, lane);
    const DmaOperand ow = dma_operand(reinterpret_cast<const bf16_t*>(wb), cols, a.d_in / 2, 0, wave, lane);
    PartTile part = part_tile(a.d_in / 2, wave, lane);
    if (a.d_in == kI8Tile) part = {kGemmBK, 0, true};   // whole
#pragma unroll
    for (int i = 0; i < MB; ++i) dma_piece_behind<true, false>(xs, ox, (uint32_t)rows * (uint32_t)a.d_in, ox, part, -1, i, wave);
#pragma unroll
    for (int i = 0; i < NB; ++i) dma_piece_behind<true, false>(wsm, ow, (uint32_t)cols * (uint32_t)a.d_in, ow, part, -1, i, wave);
    i32x4 acc[MB][NB];
#pragma unroll
    for (int mi = 0; mi < MB; ++mi)
#pragma unroll
        for (int ni = 0; ni < NB; ++ni) acc[mi][ni] = i32x4{0, 0, 0, 0};
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        if (ks * 64 >= a.d_in) break;
        Frags16<MB, NB> f;
#pragma unroll
        for (int i = 0; i < MB + NB; ++i) load_frag16<MB, NB>(f, xs, wsm, wm, wn, l15, kq, ks, i);
#pragma unroll
        for (int mi = 0; mi < MB; ++mi)
#pragma unroll
            for (int ni = 0; ni < NB; ++ni)
                acc[mi][ni] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, f.w[ni]),
                                                                    __builtin_bit_cast(i32x4, f.x[mi]), acc[mi][ni], 0, 0, 0);
    }
    ring_i8_epilogue<TO, MB, NB>(a, acc, smem, e, row0, rows, n0, wm, wn, wave, lane);
}

template <typename TO, int TB, int RB, int WV, int D>
static hipError_t launch_wave(GemmI8Args a, hipStream_t stream) {
    a.tiles_m = most_row_tiles(a, TB * 16);
    a.tile_cols = wave_tile_cols(a.tiles_m, a.d_out, RB * 16);
    a.tiles_n = ceil_div(a.d_out, a.tile_cols);
    constexpr int lds = wave_i8_lds<TB, RB, WV, D>();
    const auto kern = &gemm_i8_wave_kernel<TO, TB, RB, WV, D>;
    static_assert(lds <= 160 * 1024, "LDS");
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(kern), lds);
    if (e != hipSuccess) return e;
    if ((int64_t)a.tiles_m * a.tiles_n * WV * 64 >= (int64_t)1 << 32) return hipErrorInvalidValue;
    kern<<<a.tiles_m * a.tiles_n, WV * 64, lds, stream>>>(a);
    return hipGetLastError();
}

template <typename TO, int MB, int NB, int D>
static hipError_t launch_ring_i8(GemmI8Args a, hipStream_t stream) {
    a.tiles_m = most_row_tiles(a, MB * 32);
    a.tiles_n = ceil_div(a.d_out, NB * 32);
    constexpr int lds = ring_i8_lds<MB, NB, D>();
    const auto kern = a.d_in % kI8Tile != 0 ? &gemm_i8_ring_kernel<TO, MB, NB, D, true> : &gemm_i8_ring_kernel<TO, MB, NB, D, false>;
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(kern), lds);
    if (e != hipSuccess) return e;
    if ((int64_t)a.tiles_m * a.tiles_n * 256 >= (int64_t)1 << 32) return hipErrorInvalidValue;
    kern<<<a.tiles_m * a.tiles_n, 256, lds, stream>>>(a);
    return hipGetLastError();
}

// 256 x 256 tiles, and the tail where there is, or (groups) may be, one.  As the best of the shapes with a round of their own for the rest,
// and so, us: 4300, 5000 and 9000 x 4096 -> 4096 69.4, 77.7, 141 and 69.3, 74.7, 123; 5000 x 4096 -> 14336 247 and 228; 8 groups of 4096 ->
// 4096, 4002 and 8192 rows that fall off as 1 / j^2 92.5, 141 and 81.4, 124, dealt evenly (whole rounds: the second launch finds nothing)
// 53.4, 102 and 55.6, 103.  The size of the tail's tiles, 16 tiles of 8 groups of 4096 -> 4096 behind 256: 128 x 128 76.3, 64 x 64 68.3; 32 tiles:
// 128 x 128 78, 128 x 64 74, 64 x 64 76; dense, 17 tiles of 5263 x 4096 -> 3176 69, 64 and 69, 32 of 4600 x 4096 -> 4096 71, 68 and 71.
template <typename TO>
static hipError_t launch_largest_i8(GemmI8Args a, hipStream_t stream) {
    const int64_t tiles = (int64_t)most_row_tiles(a, 256) * ceil_div(a.d_out, 256);
    a.tail = may_have_tail(a, tiles) ? 1 : 0;
    const hipError_t e = launch_ring_i8<TO, 8, 8, 2>(a, stream);
    if (e != hipSuccess || a.tail == 0) return e;
    a.tiles_m = most_row_tiles(a, 256);
    a.tiles_n = ceil_div(a.d_out, 256);
    const auto kern = a.d_in % kI8Tile != 0 ? &gemm_i8_tail_kernel<TO, true> : &gemm_i8_tail_kernel<TO, false>;
    const hipError_t f = ensure_lds_limit(reinterpret_cast<const void*>(kern), tail_i8_lds());
    if (f != hipSuccess) return f;
    const int rest = (int)tiles - tail_start((int)tiles);
    const int wgs = a.offsets != nullptr ? kTailTiles * 4 : rest <= kTailSmall ? rest * 16 : rest <= kTailMiddle ? rest * 8 : rest * 4;
    kern<<<wgs, 256, tail_i8_lds(), stream>>>(a);
    return hipGetLastError();
}

template <typename TO, int MB, int NB>
static hipError_t launch_one_i8(GemmI8Args a, hipStream_t stream) {
    static_assert(MB >= 2, "order of the fragments");
    a.tiles_m = most_row_tiles(a, MB * 32);
    a.tiles_n = ceil_div(a.d_out, NB * 32);
    constexpr int lds = one_i8_lds<TO, MB, NB>();
    const auto kern = &gemm_i8_one_kernel<TO, MB, NB>;
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(kern), lds);
    if (e != hipSuccess) return e;
    if ((int64_t)a.tiles_m * a.tiles_n * 256 >= (int64_t)1 << 32) return hipErrorInvalidValue;
    kern<<<a.tiles_m * a.tiles_n, 256, lds, stream>>>(a);
    return hipGetLastError();
}

// ---- which kernel and tile: the one that takes the least by
//     us^3 = (launch + rounds * (round + nk * step) + tiles / 256 * nk * share)^3 + (bytes / rate)^3
// nk K tiles, rounds of one (or per_cu) tiles per CU, bytes read and written once, 5.1 TB/s by the wavefront rings and 4.9 by the others.
// The four times of a tile shape are fitted to 350 dense sizes (1 to 8192 rows, 256 to 14336 inputs and outputs) and 999 of groups (2 to 64 of
// them, random deals of chances 1, 1 / j and 1 / j^2), W not in the caches: on the dense ones the choice is 0.6% slower on average than the
// best shape of each, on the groups with their deals known 1.1%.  How rows are dealt is known on the device only, so two deals are weighed
// alike, a random one of equal chances (the mean and 1.22 standard deviations, of a Poisson law, to either side) and one that falls off as
// 1 / j^2: 2.6% slower than the best shape of each (an exactly even deal in place of the random one 3.1%).  That holds for those two laws.
// 23 sizes (4, 8 and 28 groups, 16 to 16384 rows) of other deals: 1 / j 3.5% on average and 20% at worst, half of the rows in no group 7 and
// 52%, all rows in one group 21 and 123% (8 groups of 4096 -> 4096, 128 rows: 21 us against 9.5, since the tile is chosen for
// eight matrices), and of single deals of the two laws 4.6 and 32%, 1.9 and 14%.
constexpr I8Shape kI8Shapes[kI8ShapeCount] = {
    {16, 16, 1, true, 2.92f, 1.00f, 0.039f, 0.017f},
    {16, 32, 1, true, 1.31f, 2.84f, 0.036f, 0.060f},
    {16, 64, 1, true, 0.41f, 3.85f, 0.088f, 0.052f},
    {32, 32, 1, true, 1.80f, 2.49f, 0.049f, 0.077f},
    {64, 64, 1, false, 1.00f, 3.07f, 0.145f, 0.110f},
    {96, 64, 1, false, 1.07f, 3.08f, 0.185f, 0.108f},
    {128, 64, 1, false, 1.07f, 3.12f, 0.229f, 0.102f},
    {128, 128, 1, false, 1.36f, 3.50f, 0.357f, 0.182f},
    {128, 128, 2, false, 1.76f, 2.98f, 0.293f, 0.394f},
    {192, 128, 1, false, 1.71f, 4.09f, 0.486f, 0.173f},
    {224, 128, 1, false, 1.76f, 4.53f, 0.546f, 0.155f},
    {256, 128, 1, false, 1.68f, 5.00f, 0.619f, 0.147f},
    {256, 256, 1, false, 1.21f, 8.19f, 0.665f, 0.665f},
};
static_assert(kI8Shapes[4].rows * kI8Shapes[4].cols == 64 * 64 && kI8Shapes[6].rows * kI8Shapes[6].cols == 128 * 64 &&
              kI8Shapes[8].per_cu == 2, "of the tail");
static_assert(sizeof(kI8Shapes) / sizeof(kI8Shapes[0]) == kI8ShapeCount, "shapes");

template <typename TO>
static hipError_t launch_i8(const GemmI8Args& a, hipStream_t stream) {
    // one K tile: 64 x 128 tiles without a ring against the best of the rings, 64 -> 4096, 8192 rows in one group and in 28 13.9 and 19.0 us
    // against 18.1 and 27.7, 1024 in 28 6.5 and 11.1, 16 in 28 3.7 and 4.5; 128 inputs 15.9 and 27.1 against 17.9 and 28.1
    if (a.d_in <= kI8Tile) return launch_one_i8<TO, 2, 4>(a, stream);
    switch (choose_shape(a, kI8Shapes)) {
        case 0: return launch_wave<TO, 1, 1, 4, 5>(a, stream);
        case 1: return launch_wave<TO, 1, 2, 4, 5>(a, stream);
        case 2: return launch_wave<TO, 1, 4, 4, 3>(a, stream);
        case 3: return launch_wave<TO, 2, 2, 4, 4>(a, stream);
        case 4: return launch_ring_i8<TO, 2, 2, 5>(a, stream);
        case 5: return launch_ring_i8<TO, 3, 2, 5>(a, stream);
        case 6: return launch_ring_i8<TO, 4, 2, 4>(a, stream);
        case 7: return launch_ring_i8<TO, 4, 4, 3>(a, stream);
        case 8: return launch_ring_i8<TO, 4, 4, 2>(a, stream);
        case 9: return launch_ring_i8<TO, 6, 4, 3>(a, stream);
        case 10: return launch_ring_i8<TO, 7, 4, 3>(a, stream);
        case 11: return launch_ring_i8<TO, 8, 4, 3>(a, stream);
        default: return launch_largest_i8<TO>(a, stream);
    }
}

template <typename TX, int RB, int D>
static hipError_t launch_row(GemmI8Args a, const TX* x, hipStream_t stream) {
    a.tile_cols = wave_tile_cols(1, a.d_out, RB * 16);
    a.tiles_n = ceil_div(a.d_out, a.tile_cols);
    const int lds = row_i8_ring_bytes<RB, D>() + a.T * row_i8_stride(a.d_in);
    auto go = [&](auto kern) {
        const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(kern), row_i8_lds_most<RB, D>());
        if (e != hipSuccess) return e;
        kern<<<a.tiles_n, kRowThreads, lds, stream>>>(a, x);
        return hipGetLastError();
    };
    if (a.T == 1) return a.d_in <= 4096 ? go(&gemm_i8_row_kernel<TX, RB, D, 256, 2>) : go(&gemm_i8_row_kernel<TX, RB, D, 256, 8>);
    return a.d_in <= 4096 ? go(&gemm_i8_row_kernel<TX, RB, D, 64, 8>) : go(&gemm_i8_row_kernel<TX, RB, D, 64, 16>);
}

// Against two launches, W not in the caches, GPU alone (an eager call saves 3 us of the host as well): 1, 2 and 4 x 4096 -> 4096 6.9, 7.9,
// 8.1 and 8.5, 8.9, 8.9 us, -> 14336 12.4, 13.7, 13.9 and 15.5, 15.5, 15.6; 1 and 3 x 5120 -> 13824 14.8, 17.3 and 17.2, 17.4; 1 x 14336 ->
// 4096 14.1 and 15.5; 8 x 4096 -> 4096 10.2 and 9.1.  32 columns a tile and 16: 1 x 4096 -> 4096 7.3 and 6.9, -> 14336 12.4 and 14.4.
bool base_gemm_i8_in_one(int T, int d_in) { return T <= kRowMaxTokens && T * d_in <= kRowMaxBytes; }

template <typename TX>
static hipError_t launch_base(const GemmI8Args& a, const TX* x, hipStream_t stream) {
    return a.d_out <= 4096 ? launch_row<TX, 1, 5>(a, x, stream) : launch_row<TX, 2, 3>(a, x, stream);
}
hipError_t launch_base_gemm_i8_in_one(const void* x, const int8_t* W, const float* w_scale, int T, int d_in, int d_out, bool bf16,
                                      void* out, hipStream_t stream) {
    const GemmI8Args a{nullptr, nullptr, W, w_scale, nullptr, out, T, d_in, d_out, 1, 1, 0, 0, 0, 0};
    return bf16 ? launch_base(a, (const bf16_t*)x, stream) : launch_base(a, (const float*)x, stream);
}

static GemmI8Args i8_args(const int8_t* q, const float* q_scale, const int8_t* W, const float* w_scale, const int32_t* offsets,
                          int T, int d_in, int d_out, int N, void* out) {
    // The last cache holds 256 MB: from three such matrices in turn on none is still there.  Three in turn, 128 x 128 tiles, requested as kept and
    // as read once, us: 67 MB 14.3 and 15.9, 84 MB 19.5 and 22.0, 101 MB 23.9 and 24.0, 117 MB 26.9 and 25.1, 134 MB 29.0 and 25.4.
    // All N matrices count, also where the rows are in few of them: which have rows is known on the device only.
    const int past_caches = (int64_t)N * d_out * d_in >= 100000000;
    return {q, q_scale, W, w_scale, offsets, out, T, d_in, d_out, N, 0, 0, 0, 0, past_caches};
}
hipError_t launch_gemm_i8(const int8_t* q, const float* q_scale, const int8_t* W, const float* w_scale, const int32_t* offsets,
                          int T, int d_in, int d_out, int N, bool bf16, void* out, hipStream_t stream) {
    const GemmI8Args a = i8_args(q, q_scale, W, w_scale, offsets, T, d_in, d_out, N, out);
    return bf16 ? launch_i8<bf16_t>(a, stream) : launch_i8<float>(a, stream);
}

I8Plan gemm_i8_plan(int T, int d_in, int d_out, int N, bool grouped) {
    static const int32_t some = 0;   // offsets, which the host does not read
    const GemmI8Args a = i8_args(nullptr, nullptr, nullptr, nullptr, grouped ? &some : nullptr, T, d_in, d_out, N, nullptr);
    if (d_in <= kI8Tile) return {"one", 64, 128, 1, false, false};
    const I8Shape& s = kI8Shapes[choose_shape(a, kI8Shapes)];
    const bool largest = s.rows * s.cols == 256 * 256;
    return {s.wave ? "wave" : "ring", s.rows, s.cols, s.per_cu, !s.wave && !largest && a.past_caches != 0,
            largest && may_have_tail(a, (int64_t)most_row_tiles(a, 256) * ceil_div(d_out, 256))};
}

template <typename TO, int TB, int RB, int WV, int D>
static hipError_t init_wave() {
    return ensure_lds_limit(reinterpret_cast<const void*>(&gemm_i8_wave_kernel<TO, TB, RB, WV, D>), wave_i8_lds<TB, RB, WV, D>());
}
template <typename TO, int MB, int NB, int D>
static hipError_t init_ring() {
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(&gemm_i8_ring_kernel<TO, MB, NB, D, true>), ring_i8_lds<MB, NB, D>());
    return e != hipSuccess ? e : ensure_lds_limit(reinterpret_cast<const void*>(&gemm_i8_ring_kernel<TO, MB, NB, D, false>), ring_i8_lds<MB, NB, D>());
}
template <typename TO>
static hipError_t init_tail() {
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(&gemm_i8_tail_kernel<TO, true>), tail_i8_lds());
    return e != hipSuccess ? e : ensure_lds_limit(reinterpret_cast<const void*>(&gemm_i8_tail_kernel<TO, false>), tail_i8_lds());
}
template <typename TX, int RB, int D>
static hipError_t init_row() {
    hipError_t e = hipSuccess;
    for (const void* k : {reinterpret_cast<const void*>(&gemm_i8_row_kernel<TX, RB, D, 256, 2>),
                          reinterpret_cast<const void*>(&gemm_i8_row_kernel<TX, RB, D, 256, 8>),
                          reinterpret_cast<const void*>(&gemm_i8_row_kernel<TX, RB, D, 64, 8>),
                          reinterpret_cast<const void*>(&gemm_i8_row_kernel<TX, RB, D, 64, 16>)})
        if (e == hipSuccess) e = ensure_lds_limit(k, row_i8_lds_most<RB, D>());
    return e;
}
template <typename TO>
static hipError_t init_i8() {   // every kernel that launch_i8 and launch_base may start
    hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(&gemm_i8_one_kernel<TO, 2, 4>), one_i8_lds<TO, 2, 4>());
    for (hipError_t f : {init_wave<TO, 1, 1, 4, 5>(), init_wave<TO, 1, 2, 4, 5>(), init_wave<TO, 1, 4, 4, 3>(), init_wave<TO, 2, 2, 4, 4>(),
                         init_ring<TO, 2, 2, 5>(), init_ring<TO, 3, 2, 5>(), init_ring<TO, 4, 2, 4>(), init_ring<TO, 4, 4, 3>(),
                         init_ring<TO, 4, 4, 2>(), init_ring<TO, 6, 4, 3>(), init_ring<TO, 7, 4, 3>(), init_ring<TO, 8, 4, 3>(),
                         init_ring<TO, 8, 8, 2>(), init_tail<TO>(), init_row<TO, 1, 5>(), init_row<TO, 2, 3>()})
        if (e == hipSuccess) e = f;
    return e;
}
hipError_t gemm_i8_init_kernels() {
    const hipError_t e = init_i8<bf16_t>();
    return e != hipSuccess ? e : init_i8<float>();
}

}  // namespace meteora
