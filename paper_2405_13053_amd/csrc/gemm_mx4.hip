// Products of 4-bit values with a scale for every 32 inputs (see quant_mx4.hpp), over groups of consecutive rows:
//
//     out[t,c] = sum_b 2^(Eq[t,b] + Ew[e,c,b] - 254) sum_{i in block b} q[t,i] * W_e[c,i],     offsets[e] <= t < offsets[e+1]
//
// fp32 sums, one rounding to bf16 where the output is that.  v_mfma_scale_f32_16x16x128_f8f6f4 takes 16 bytes a lane and operand, 32
// values of one block, and the block's scale byte from a register beside them: a K tile of 128 bytes a row is 256 inputs and two
// instructions, and takes as many bytes and cycles as 128 inputs do in 8 bits and 64 in bf16.  So these are the schedules of the 8-bit
// products (see gemm_i8.hip) with the scales as a third operand.  Lane kq * 16 + l15 holds row l15 and block kq of an instruction's four;
// the word of scales that it needs for 512 inputs is bytes kq * 4 .. + 3 of the row's 16, and 16 rows' words are 256 bytes on end.
//
// gemm_mx4_ring_kernel   many rows: tiles of 64 x 64 to 256 x 256, rings of LDS slots, scales in registers with two slots, in the slots of deeper rings
// gemm_mx4_wave_kernel   few rows: a ring to every wavefront, scales in its slots
// gemm_mx4_one_kernel    up to 256 inputs: no ring
// gemm_mx4_row_kernel    up to 16 tokens of meteora_base_gemm_mx4: their quantisation too
#include "common.hpp"
#include "gemm_mfma.hpp"
#include "gemm_rows.hpp"
#include "kernels.hpp"
#include "quant_mx4.hpp"

namespace meteora {

using GemmMx4Args = GemmRowsArgs<uint8_t>;   // q_scale[chunks][T][16], w_scale[N][chunks][d_out][16]; chunks of 512 inputs, 256 bytes
typedef __attribute__((ext_vector_type(8))) int32_t i32x8;

// The product of two fragments; byte KS of each word is the scale.
template <int KS>
__device__ __forceinline__ f32x4 mfma_mx4(const u32x4& w, const u32x4& x, const f32x4& acc, uint32_t sw, uint32_t sx) {
    const i32x8 a{(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0}, b{(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, KS, (int)sw, KS, (int)sx);
}
template <int KS>
__device__ __forceinline__ void mfma16_mx4(f32x4& acc, const bf16x8& w, const bf16x8& x, uint32_t sw, uint32_t sx) {
    if constexpr (KS == 0)
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                     : "+a"(acc) : "v"(w), "v"(x), "v"(sw), "v"(sx));
    else
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                     : "+a"(acc) : "v"(w), "v"(x), "v"(sw), "v"(sx));
}

template <int TB, int RB, int WV, int D>
constexpr int wave_mx4_lds() {
    constexpr int ring = WV * D * (TB + RB) * 2304, sums = WV * TB * RB * 1024;
    return ring > sums ? ring : sums;
}

// The wavefronts' tiles are added in LDS ([wave][block][lane]) and leave as rows.  W is the first operand, so a lane holds 4
// consecutive columns of row l15 of a block
template <typename TO, int TB, int RB, int WV>
__device__ __forceinline__ void wave_mx4_sums(const GemmMx4Args& a, const f32x4 (&acc)[TB][RB], unsigned char* smem, int row0, int rows, int n0, int cols, int wave, int lane) {
    const int l15 = lane & 15, kq = lane >> 4;
    f32x4* part = reinterpret_cast<f32x4*>(smem);
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int r = 0; r < RB; ++r) part[(wave * TB * RB + t * RB + r) * 64 + lane] = acc[t][r];
    __syncthreads();
    constexpr int OUT = (TB * RB + WV - 1) / WV;
#pragma unroll
    for (int u = 0; u < OUT; ++u) {
        const int b = wave + u * WV;
        const int row = b / RB * 16 + l15, col = b % RB * 16 + kq * 4;   // d_out % 8 == 0: 4 columns are all in or all out
        if (b >= TB * RB || row >= rows || col >= cols) continue;
        f32x4 sum = part[b * 64 + lane];
#pragma unroll
        for (int v = 1; v < WV; ++v) sum += part[(v * TB * RB + b) * 64 + lane];
        const float v[4] = {sum[0], sum[1], sum[2], sum[3]};
        store4((TO*)a.out + (size_t)(row0 + row) * a.d_out + n0 + col, v);
    }
}

// Few rows: TB x 16 rows of q, RB x 16 rows of W, WV wavefronts, each with every WV-th K tile of 256 inputs and a ring of its own of
// D slots, so that no wavefront waits for another before the end.
template <typename TO, int TB, int RB, int WV, int D>
__global__ __launch_bounds__(WV * 64) void gemm_mx4_wave_kernel(const GemmMx4Args a) {
    constexpr int NX = 2 * TB, NW = 2 * RB, NS = TB + RB, NL = NX + NW + NS;   // load instructions per K tile: 8 rows each, 16 rows' scales
    constexpr int NM = 2 * TB * RB;                         // MFMAs per K tile
    constexpr int kSlot = (TB + RB) * 2304;                 // a K tile and its scales
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
    unsigned char* const ring = smem + wave * D * kSlot;

    WaveOperand<TB> x(a.q + (size_t)row0 * ld, rows, ld, lane);
    WaveOperand<RB> w(a.W + ((size_t)e * a.d_out + n0) * ld, cols, ld, lane);
    const ScaleRows xs(a.q_scale, a.T, row0, rows, a.d_in);
    const ScaleRows ws(a.w_scale + (size_t)e * mx4_scale_bytes(a.d_out, a.d_in * 2), a.d_out, n0, cols, a.d_in);
    const uint32_t at_scale = (uint32_t)l15 * 16 + kq * 4;
    const int nk = ceil_div(a.d_in, 128), n = wave < nk ? (nk - 1 - wave) / WV + 1 : 0;
    __amdgpu_buffer_rsrc_t xsr, wsr;
    auto at_tile = [&](int kt) {
        x.at_tile(kt, nk);
        w.at_tile(kt, nk);
        xsr = xs.chunk(kt >> 1);
        wsr = ws.chunk(kt >> 1);
    };
    auto request = [&](unsigned char* slot, int i) {   // load i of that K tile: W's first
        if (i < NW) w.template request<kReadOnceI8>(slot, i);
        else if (i < NW + NX) x.template request<0>(slot + NW * 1024, i - NW);
        else if (i < NW + NX + RB) mx4_scale_lds(wsr, slot + (TB + RB) * 2048 + (i - NW - NX) * 256, at_scale + (i - NW - NX) * 256);
        else mx4_scale_lds(xsr, slot + (TB + RB) * 2048 + (i - NW - NX) * 256, at_scale + (i - NW - NX - RB) * 256);
    };
#pragma unroll
    for (int d = 0; d < D; ++d) {
        at_tile(wave + d * WV);
#pragma unroll
        for (int i = 0; i < NL; ++i) request(ring + d * kSlot, i);
    }
    f32x4 acc[TB][RB];
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int r = 0; r < RB; ++r) acc[t][r] = f32x4{0.f, 0.f, 0.f, 0.f};
    // the scales of this wavefront's K tiles, all even ones or all odd ones, are the low or the high half of their words
    static_assert(WV % 2 == 0, "K tiles of a wavefront");
    const int half = (wave & 1) * 16;
    struct Frag { u32x4 x[2][TB], w[2][RB]; uint32_t sx[TB], sw[RB]; };
    auto read = [&](Frag& f, const unsigned char* slot) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const int at = l15 * 128 + swz(l15, ks * 4 + kq) * 16;   // row l15 of a block of 16
#pragma unroll
            for (int r = 0; r < RB; ++r) f.w[ks][r] = *reinterpret_cast<const u32x4*>(slot + r * 2048 + at);
#pragma unroll
            for (int t = 0; t < TB; ++t) f.x[ks][t] = *reinterpret_cast<const u32x4*>(slot + (RB + t) * 2048 + at);
        }
        const unsigned char* const words = slot + (TB + RB) * 2048 + lane * 4;
#pragma unroll
        for (int r = 0; r < RB; ++r) f.sw[r] = *reinterpret_cast<const uint32_t*>(words + r * 256) >> half;
#pragma unroll
        for (int t = 0; t < TB; ++t) f.sx[t] = *reinterpret_cast<const uint32_t*>(words + (RB + t) * 256) >> half;
    };
    int slot = 0, kt = wave + D * WV;   // of the tile that is multiplied; the one that is requested
    // multiplies `cur` while `nxt` is read and the tile D ahead is requested into the slot that cur came from
    auto step = [&](Frag& cur, Frag& nxt) {
        unsigned char* const mine = ring + slot * kSlot;
        slot = slot + 1 == D ? 0 : slot + 1;
        // the next tile has landed: of the loads only those of the D - 2 tiles behind it may be in flight; cur has left its slot
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((D - 2) * NL) : "memory");
        read(nxt, ring + slot * kSlot);
        at_tile(kt);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            request(mine, i);
#pragma unroll
            for (int m = i * NM / NL; m < (i + 1) * NM / NL; ++m) {
                const int ks = m / (TB * RB), t = m / RB % TB, r = m % RB;
                acc[t][r] = ks == 0 ? mfma_mx4<0>(cur.w[0][r], cur.x[0][t], acc[t][r], cur.sw[r], cur.sx[t])
                                    : mfma_mx4<1>(cur.w[1][r], cur.x[1][t], acc[t][r], cur.sw[r], cur.sx[t]);
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

    wave_mx4_sums<TO, TB, RB, WV>(a, acc, smem, row0, rows, n0, cols, wave, lane);
}

// ------------------------------------------------------------------------------------------
// A few tokens and their quantisation in one launch (meteora_base_gemm_mx4): every workgroup quantises all of x itself, into LDS, while its
// first tiles of W are on their way, which costs less than a launch in front (graphs of calls, weights in turn): 1, 2, 4 and 8 tokens of 4096 -> 4096 4.7,
// 5.3, 5.5 and 7.7 us, with quantize_mx4_kernel in front 6.9, 6.8, 6.9 and 7.0 and a launch more for the host; 16 of 1024 -> 4096 4.8 and 6.1; 4 and 6 of
// 5120 -> 5120 8.5 and 8.9, and 8.5 and 8.6; 3 and 4 of 4096 -> 14336, where workgroups follow one another on a CU, 10.0 and 12.2, and 11.2 and 11.0.
// W goes through the wavefronts' rings as above; a lane without a row of its own multiplies another's, and its result is not kept.
// ------------------------------------------------------------------------------------------
constexpr int kRowThreads = 256, kRowMaxTokens = 16, kRowHeld = 18, kRowMaxInputs = kRowHeld * kRowThreads * 8;   // of all tokens, in whole chunks
constexpr int row_mx4_stride(int d) { return (d / 2 + 127) / 128 * 128 + 16; }   // bytes; rows start 4 banks apart
constexpr int row_mx4_bytes(int T, int d) { return T * (row_mx4_stride(d) + mx4_chunks(d) * 16); }
template <int RB, int D>
constexpr int row_mx4_ring_bytes() { return 4 * D * RB * 2304; }   // and the sums in its place
template <int RB, int D>
constexpr int row_mx4_lds_most() { return row_mx4_ring_bytes<RB, D>() + kRowMaxInputs / 2 + kRowMaxTokens * (127 + 16) + kRowMaxInputs / 32; }

// HELD: pieces of 8 inputs to a thread
template <typename TX, int RB, int D, int HELD>
__global__ __launch_bounds__(kRowThreads) void gemm_mx4_row_kernel(const GemmMx4Args a, const TX* __restrict__ x) {
    constexpr int WV = 4, NL = 3 * RB;
    static_assert(D >= 2 && (D - 1) * NL < 64, "vmcnt");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, kq = lane >> 4;
    const int n0 = xcd_order(blockIdx.x, a.tiles_n) * a.tile_cols, cols = min(a.tile_cols, a.d_out - n0);
    const uint32_t ld = (uint32_t)a.d_in;
    unsigned char* const ring = smem + wave * D * RB * 2304;
    unsigned char* const xq = smem + row_mx4_ring_bytes<RB, D>();
    const int inputs = a.d_in * 2, per = inputs / 8, chunks = mx4_chunks(inputs), stride = row_mx4_stride(inputs);
    unsigned char* const xs = xq + a.T * stride;   // [T][chunks][16]

    // whole chunks of 64 pieces, a block to a quad of threads; those past the last input are zeros with scale 0, since whatever LDS held there
    // might be a NaN
    Piece8<TX> held[HELD];
    const int pieces = chunks * 64;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int p = i * kRowThreads + tid, t = p / pieces, j = p - t * pieces;
        held[i] = Piece8<TX>{};
        if (t < a.T && j < per) held[i].load(x + (size_t)t * inputs + j * 8);
    }
    WaveOperand<RB> w(a.W + (size_t)n0 * ld, cols, ld, lane);
    const ScaleRows ws(a.w_scale, a.d_out, n0, cols, a.d_in);
    const uint32_t at_scale = (uint32_t)l15 * 16 + kq * 4;
    const int nk = ceil_div(a.d_in, 128), n = wave < nk ? (nk - 1 - wave) / WV + 1 : 0;
    auto request = [&](unsigned char* slot, int kt) {
        w.at_tile(kt, nk);
        const auto scales = ws.chunk(kt >> 1);
#pragma unroll
        for (int i = 0; i < 2 * RB; ++i) w.template request<kReadOnceI8>(slot, i);
#pragma unroll
        for (int r = 0; r < RB; ++r) mx4_scale_lds(scales, slot + RB * 2048 + r * 256, at_scale + r * 256);
    };
#pragma unroll
    for (int d = 0; d < D; ++d) request(ring + d * RB * 2304, wave + d * WV);
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int p = i * kRowThreads + tid, t = p / pieces, j = p - t * pieces, b = j >> 2;
        const uint32_t E = mx4_exponent(held[i]), v = mx4_quantize8(held[i], E);
        if (t >= a.T) continue;
        if (j < per) *reinterpret_cast<uint32_t*>(xq + t * stride + j * 4) = v;
        if ((j & 3) == 0) xs[t * chunks * 16 + (b >> 4) * 16 + (b & 3) * 4 + ((b & 15) >> 2)] = (uint8_t)E;
    }
    __syncthreads();
    const unsigned char* const mine = xq + (l15 % a.T) * stride;
    const unsigned char* const my_scales = xs + (l15 % a.T) * chunks * 16 + kq * 4 + (wave & 1) * 2;   // a wavefront's K tiles are all even or all odd
    const int half = (wave & 1) * 16;

    f32x4 acc[1][RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) acc[0][r] = f32x4{0.f, 0.f, 0.f, 0.f};
    int slot = 0;
    for (int i = 0; i < n; ++i) {
        const int kt = wave + i * WV;
        const unsigned char* const at = ring + slot * RB * 2304;
        // of the loads only those of the D - 1 tiles behind this one may be in flight
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * NL) : "memory");
        u32x4 wf[2][RB], xf[2];
        uint32_t sw[RB];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
            for (int r = 0; r < RB; ++r) wf[ks][r] = *reinterpret_cast<const u32x4*>(at + r * 2048 + l15 * 128 + swz(l15, ks * 4 + kq) * 16);
            xf[ks] = *reinterpret_cast<const u32x4*>(mine + kt * 128 + (ks * 4 + kq) * 16);   // past the last input: any codes, times zeros
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) sw[r] = *reinterpret_cast<const uint32_t*>(at + RB * 2048 + r * 256 + lane * 4) >> half;
        const uint32_t sx = *reinterpret_cast<const uint16_t*>(my_scales + (kt >> 1) * 16);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slot is read
        request(ring + slot * RB * 2304, kt + D * WV);
        slot = slot + 1 == D ? 0 : slot + 1;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            acc[0][r] = mfma_mx4<0>(wf[0][r], xf[0], acc[0][r], sw[r], sx);
            acc[0][r] = mfma_mx4<1>(wf[1][r], xf[1], acc[0][r], sw[r], sx);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may land in what follows
    __syncthreads();
    wave_mx4_sums<TX, 1, RB, WV>(a, acc, smem, 0, a.T, n0, cols, wave, lane);
}

// Many rows: the schedule of gemm_i8_ring_kernel.  The instruction is in assembly with its accumulator tied, with the same care
// (tests/test_mfma_waits_mx4_host.py reads the compiled code).  Scales: with rings of two slots, which take all of LDS with 256 x 256 tiles, words in
// registers, MB + NB a lane for two K tiles, loaded a tile and a half ahead: 64 rows' 16 bytes to an instruction, a row to a lane, and turned to
// the words of four blocks of rows in registers (turn_scales); the second tile's are shifted down.  A load for every block of 16 rows
// instead, 16 a wavefront rather than 4, held up the K tiles' own: 4096 x 4096 -> 4096 34.8 us, 8192 x 4096 -> 14336 240.  Loads complete in order, so in
// deeper rings those words would wait for every K tile requested before them; there the scales are part of the slots, 16 bytes a row
// (those of two K tiles, in either's slot), 64 rows a load instruction.
// In: lane g * 16 + l has the 16 bytes of row g * 16 + l, a word for each quarter.  Out: word i of lane kq * 16 + l is word kq of row i * 16 + l.
__device__ __forceinline__ void turn_scales(const u32x4& v, uint32_t (&out)[4]) {
    const auto a = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false), b = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    out[0] = c[0];
    out[1] = c[1];
    out[2] = d[0];
    out[3] = d[1];
}
template <int BLOCKS, int D>
constexpr int mx4_slot_bytes() { return BLOCKS * 32 * kI8Tile + (D > 2 ? ceil_div(BLOCKS, 2) * 1024 : 0); }
template <int MB, int NB, int D>
constexpr int ring_mx4_lds() {
    constexpr int ring = D * mx4_slot_bytes<MB, D>() + (D + 1) * mx4_slot_bytes<NB, D>(), stage = 4 * 32 * (NB * 64 + 16);
    return ring > stage ? ring : stage;
}

// The tile leaves by way of LDS, 32 (16) rows a wavefront at a time, so that stores are 16-byte pieces of whole rows.  Through the L2,
// see kWriteThrough.  KEPT: where rows are no whole lines they stay in the L2 until the neighbouring tile's part is there; written through, a line
// goes to memory in two parts.  That is worth it in gemm_mx4_one_kernel (5195 x 96 -> 13200 31.6 and 69.7 us, 8192 x 64 -> 4104 18.0 and 23.2), whose
// four or five workgroups to a CU all store at once, not behind rings, however short: kept and written through, 4096 x 288, 512 and 1024 -> 4104 19.0, 19.1 and
// 22.3, and 17.1, 17.1 and 20.8; 8192 x 288 and 768 -> 13200 72 and 84, and 69 and 81; 1000 x 288 -> 13200 14.1 and 12.2; fp32, 4096 x 288 -> 4104 22.5 and 21.0.
template <typename TO, int MB, int NB, bool KEPT>
__device__ __forceinline__ void ring_mx4_epilogue(const GemmMx4Args& a, f32x4 (&acc)[MB][NB], unsigned char* smem, int e, int row0,
                                                 int rows, int n0, int wm, int wn, int wave, int lane) {
    constexpr int EB = sizeof(TO), RS = MB % 2 == 0 ? 32 : 16;
    constexpr int EST = NB * 16 * EB + 16, PPR = NB * EB, NP = RS * PPR / 64;   // bytes and pieces per staged row, pieces per lane
    static_assert(RS * PPR % 64 == 0, "whole wavefronts of pieces");
    const int l15 = lane & 15, kq = lane >> 4;
    __syncthreads();   // every wavefront is done with the operand tiles
    unsigned char* ep = smem + wave * RS * EST;
    const uint32_t row_bytes = (uint32_t)a.d_out * EB;
    const bool whole = row_bytes % 128 == 0;   // all of a line is this tile's
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
                const float v[4] = {acc[mb + h][nb][0], acc[mb + h][nb][1], acc[mb + h][nb][2], acc[mb + h][nb][3]};
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
            if (!KEPT || whole) __builtin_amdgcn_raw_buffer_store_b128(v, out, at, 0, kWriteThrough);
            else __builtin_amdgcn_raw_buffer_store_b128(v, out, at, 0, 0);
        }
        sync();
        __builtin_amdgcn_sched_barrier(0);   // accumulators leave their registers 32 rows at a time
    }
}

// One tile.  PART: d_in may end in a partial K tile.  ONCE: no other workgroup reads these rows of W.
template <typename TO, int MB, int NB, int D, bool PART, bool ONCE>
__device__ __forceinline__ void ring_mx4_tile(const GemmMx4Args& a, unsigned char* smem, int e, int row0, int rows, int n0) {
    constexpr int BM = MB * 32, BN = NB * 32, PX = MB, PW = NB;   // 2 x 2 wavefronts; load instructions per wavefront and tile
    constexpr bool SLOTS = D > 2;                                 // scales in the slots
    constexpr int GX = ceil_div(BM, 64), GW = ceil_div(BN, 64), PS = SLOTS ? ceil_div(GX + GW, 4) : 0, P = PX + PW + PS;
    static_assert((NB % 2 == 0 || MB % 2 == 0) && D >= 2 && D <= 5 && (D - 1) * P < 64, "2 x 2 micro-blocks; vmcnt");
    constexpr int NR = MB + NB, NM = MB * NB;   // fragment reads and MFMAs per k-step of 128
    constexpr int RA = NM * 3 / 4 / NR > 0 ? NM * 3 / 4 / NR : 1, RB = NM / NR;   // MFMAs per read, see the bf16 kernel
    static_assert(RB >= 1, "a k-step needs one MFMA per fragment read");
    bf16_t* ring = reinterpret_cast<bf16_t*>(smem);
    constexpr int kXElems = mx4_slot_bytes<MB, D>() / 2, kWElems = mx4_slot_bytes<NB, D>() / 2;   // of two bytes, as everything that is shared

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

    // Scales: the low half of a word is the tile's that is multiplied; next: of the chunk of two tiles behind it, or of the tile
    const ScaleRows xsc(a.q_scale, a.T, row0, rows, a.d_in);
    const ScaleRows wsc(a.w_scale + (size_t)e * mx4_scale_bytes(a.d_out, a.d_in * 2), a.d_out, n0, cols, a.d_in);
    constexpr int SX = ceil_div(MB, 4), SW = ceil_div(NB, 4);
    uint32_t sx[SX * 4], sw[SW * 4], sx_next[SX * 4], sw_next[SW * 4];
    u32x4 ahead[SX + SW];
    auto request_ahead = [&](int chunk, int i) {   // i < SX + SW
        const int r = i < SX ? wm + i * 64 : wn + (i - SX) * 64;
        ahead[i] = __builtin_amdgcn_raw_buffer_load_b128((i < SX ? xsc : wsc).chunk(chunk), (uint32_t)(r + lane) * 16, 0, 0);
    };
    auto take_ahead = [&] {
#pragma unroll
        for (int i = 0; i < SX; ++i) turn_scales(ahead[i], *reinterpret_cast<uint32_t(*)[4]>(sx + i * 4));
#pragma unroll
        for (int i = 0; i < SW; ++i) turn_scales(ahead[SX + i], *reinterpret_cast<uint32_t(*)[4]>(sw + i * 4));
    };
    if constexpr (!SLOTS) {
#pragma unroll
        for (int i = 0; i < SX + SW; ++i) request_ahead(0, i);
    }
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
    auto request_s = [&](bf16_t* xsl, bf16_t* wsl, int kt) {   // 64 rows each; fewer than there are wavefronts: some twice
#pragma unroll
        for (int j = 0; j < PS; ++j) {
            const int g = (j * 4 + wave) % (GX + GW), r = g < GX ? g : g - GX;
            const __amdgpu_buffer_rsrc_t rsrc = (g < GX ? xsc : wsc).chunk(kt >> 1);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rsrc, (__attribute__((address_space(3))) void*)((g < GX ? xsl + BM * kGemmBK : wsl + BN * kGemmBK) + r * 512), 16,
                (uint32_t)(r * 64 + lane) * 16, 0, 0, 0);
        }
    };
    auto read_scales = [&](uint32_t (&tx)[SX * 4], uint32_t (&tw)[SW * 4], const bf16_t* xsl, const bf16_t* wsl, int kt) {
        const int half = kt & 1;
#pragma unroll
        for (int i = 0; i < MB; ++i)
            tx[i] = *reinterpret_cast<const uint16_t*>(xsl + BM * kGemmBK + (wm + i * 16 + l15) * 8 + kq * 2 + half);
#pragma unroll
        for (int i = 0; i < NB; ++i)
            tw[i] = *reinterpret_cast<const uint16_t*>(wsl + BN * kGemmBK + (wn + i * 16 + l15) * 8 + kq * 2 + half);
    };
    auto request_tile = [&](int it, auto is_part) {
#pragma unroll
        for (int i = 0; i < PX; ++i) request_x(xslot(it), it, i, is_part);
#pragma unroll
        for (int i = 0; i < PW; ++i) request_w(wslot(it), it, i, is_part);
        request_s(xslot(it), wslot(it), it);
    };
#pragma unroll
    for (int t = 0; t < D; ++t)
        if (t < nk_main) request_tile(t, std::false_type{});
    if (PART && nk_main < D && nk > nk_main) request_tile(nk_main, std::true_type{});
    f32x4 acc[MB][NB];   // first values while the first tile is on its way; two wait states or more before the first MFMA
#pragma unroll
    for (int mi = 0; mi < MB; ++mi)
#pragma unroll
        for (int ni = 0; ni < NB; ++ni) {
            acc[mi][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
            asm volatile("" : "+a"(acc[mi][ni]));
        }
    asm volatile("s_nop 1" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);

    Frags16<MB, NB> f0, f1;
    auto wait_tiles = [&](int left) {   // the loads of at most `left` tiles may still be in flight
        if (D > 4 && left >= 4) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(D > 4 ? 4 * P : 0) : "memory");
        else if (D > 3 && left == 3) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(D > 3 ? 3 * P : 0) : "memory");
        else if (D > 2 && left == 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(D > 2 ? 2 * P : 0) : "memory");
        else if (left == 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(P) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    wait_tiles(min(nk, D) - 1);   // d_in >= 16: one K tile at least
#pragma unroll
    for (int i = 0; i < NR; ++i) load_frag16<MB, NB>(f0, xslot(0), wslot(0), wm, wn, l15, kq, 0, i);
    if constexpr (SLOTS) {
        read_scales(sx, sw, xslot(0), wslot(0), 0);
    } else {
        take_ahead();
        asm volatile("s_nop 1" ::: "memory");
    }
    __builtin_amdgcn_sched_barrier(0);

    using K0 = std::integral_constant<int, 0>;
    using K1 = std::integral_constant<int, 1>;
    auto mfmas = [&](const Frags16<MB, NB>& f, int k0, int k1, auto ks) {
#pragma unroll
        for (int k = k0; k < k1; ++k)
            mfma16_mx4<decltype(ks)::value>(acc[order_mi<MB, NB>(k)][order_ni<MB, NB>(k)], f.w[order_ni<MB, NB>(k)], f.x[order_mi<MB, NB>(k)],
                                            sw[order_ni<MB, NB>(k)], sx[order_mi<MB, NB>(k)]);
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
        int issued = 0, scale_piece = 0;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            mfmas(f0, i * RA, (i + 1) * RA, K0{});
            load_frag16<MB, NB>(f1, xs, ws, wm, wn, l15, kq, 1, i);
            if constexpr (REQ < 2) {
#pragma unroll
                for (int c = 0; c < pieces_after_read(i, PW, NR); ++c) request_w(wreq, it + D, issued++, IsPart{});
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        mfmas(f0, NR * RA, NM, K0{});
        __builtin_amdgcn_sched_barrier(0);
        // tile it + 1 must have landed, and every wavefront's reads of tile it must be complete
        if constexpr (REQ < 2)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(PW + (D - 2) * P) : "memory");
        else
            wait_tiles(nk - 2 - it);
        const bool odd = PH >= 0 ? PH % 2 != 0 : (it & 1) != 0;
        if constexpr (SLOTS) read_scales(sx_next, sw_next, xsl(1), wsl(1), it + 1);   // behind the last tile: of no use
        else if (PH < 0 && !odd) {
#pragma unroll
            for (int i = 0; i < SX + SW; ++i) request_ahead((it >> 1) + 1, i);
        }
        __builtin_amdgcn_sched_barrier(0);
        // k-step 1: its MFMAs, the first fragments of tile it + 1 and the row pieces of tile it + D into the slot just drained
        const bf16_t* xn = xsl(1);
        const bf16_t* wnx = wsl(1);
        if constexpr (REQ < 2) {
            issued = 0;
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                mfmas(f1, i * RB, (i + 1) * RB, K1{});
                load_frag16<MB, NB>(f0, xn, wnx, wm, wn, l15, kq, 0, i);
#pragma unroll
                for (int c = 0; c < pieces_after_read(i, PX, NR); ++c) request_x(xreq, it + D, issued++, IsPart{});
                if constexpr (!SLOTS && PH >= 0 && PH % 2 == 0) {
#pragma unroll
                    for (int c = 0; c < pieces_after_read(i, SX + SW, NR); ++c) request_ahead((it >> 1) + 1, scale_piece++);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            request_s(xreq, wreq, it + D);
            __builtin_amdgcn_sched_barrier(0);
            mfmas(f1, NR * RB, NM, K1{});
        } else {
            if (it + 1 < nk) {   // reads only: MFMAs in both arms of a branch make the compiler copy accumulators
#pragma unroll
                for (int i = 0; i < NR; ++i) load_frag16<MB, NB>(f0, xn, wnx, wm, wn, l15, kq, 0, i);
            }
            __builtin_amdgcn_sched_barrier(0);
            mfmas(f1, 0, NM, K1{});
        }
        if constexpr (SLOTS) {
#pragma unroll
            for (int i = 0; i < MB; ++i) sx[i] = sx_next[i];
#pragma unroll
            for (int i = 0; i < NB; ++i) sw[i] = sw_next[i];
        } else if (odd) {
            take_ahead();
        } else {
#pragma unroll
            for (int i = 0; i < MB; ++i) sx[i] >>= 16;
#pragma unroll
            for (int i = 0; i < NB; ++i) sw[i] >>= 16;
        }
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_nop 1" ::: "memory");   // wait states between these and an MFMA
        if constexpr (PH < 0) {
            slot_x = (int)(xn - ring);
            slot_w = (int)(wnx - ring);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    using Req0 = std::integral_constant<int, 0>;
    using Rt = std::integral_constant<int, -1>;
    int it = 0;
    constexpr int TRIP = D * (D + 1);   // a whole period of both rings, an even number: no slot arithmetic between two tiles
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
    ring_mx4_epilogue<TO, MB, NB, false>(a, acc, smem, e, row0, rows, n0, wm, wn, wave, lane);
}

// Two copies of the loop for the two policies of W's loads, see gemm_mx4_ring_kernel.
template <typename TO, int MB, int NB, int D, bool PART>
__global__ __launch_bounds__(256) void gemm_mx4_ring_kernel(const GemmMx4Args a) {
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
            ring_mx4_tile<TO, MB, NB, D, PART, true>(a, smem, rt.e, rt.row0, rt.rows, tile_n * BN);
            return;
        }
    ring_mx4_tile<TO, MB, NB, D, PART, false>(a, smem, rt.e, rt.row0, rt.rows, tile_n * BN);
}

// The 256 x 256 tiles behind tail_start, in smaller ones: as small as one to a CU allows, or two of the largest.  The number of tiles of
// groups is known here only, and so is their size.
template <typename TO, int MB, int NB, int D, bool PART>
__device__ __forceinline__ void tail_mx4_part(const GemmMx4Args& a, const RowTiles<256>& row_tiles, unsigned char* smem, int first, int tiles) {
    constexpr int BM = MB * 32, BN = NB * 32, PM = 256 / BM, PN = 256 / BN;
    const int id = first + (int)blockIdx.x / (PM * PN), m0 = (int)blockIdx.x % PM * BM;
    if (id >= tiles) return;
    int tile_m, tile_n;
    tile_of_workgroup(id, row_tiles.count, a.tiles_n, tile_m, tile_n);
    const RowTile rt = row_tiles.at(a, tile_m);
    const int rows = min(BM, rt.rows - m0), n0 = tile_n * 256 + (int)blockIdx.x / PM % PN * BN;
    if (rows <= 0 || n0 >= a.d_out) return;
    ring_mx4_tile<TO, MB, NB, D, PART, false>(a, smem, rt.e, rt.row0 + m0, rows, n0);
}
constexpr int tail_mx4_lds() {   // two workgroups to a CU
    const int a = ring_mx4_lds<2, 2, 3>(), b = ring_mx4_lds<4, 2, 2>(), c = ring_mx4_lds<4, 4, 2>();
    return a > b ? (a > c ? a : c) : (b > c ? b : c);
}
static_assert(2 * tail_mx4_lds() <= 160 * 1024, "LDS");

template <typename TO, bool PART>
__global__ __launch_bounds__(256) void gemm_mx4_tail_kernel(const GemmMx4Args a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const RowTiles<256> row_tiles(a, (int)threadIdx.x & 63);
    const int tiles = row_tiles.count * a.tiles_n, first = tail_start(tiles);
    if (tiles - first <= kTailSmall) tail_mx4_part<TO, 2, 2, 3, PART>(a, row_tiles, smem, first, tiles);
    else if (tiles - first <= kTailMiddle) tail_mx4_part<TO, 4, 2, 2, PART>(a, row_tiles, smem, first, tiles);
    else tail_mx4_part<TO, 4, 4, 2, PART>(a, row_tiles, smem, first, tiles);
}

// Up to 256 inputs (the expand of adapters): one K tile, and the output is what there is to move.  The same tiles without a ring, so
// that four or five workgroups share a CU and one's loads and arithmetic lie under another's stores.  4096 x 256 -> 4096 9.8 us, with rings of 64 x 64 and
// 128 x 128 32.3 and 10.6; 8192 x 128 -> 4096 14.2, 65.3 and 17.8; 16384 x 64 -> 4096 25.4 (5.4 TB/s), 129 and 31.0.
template <typename TO, int MB, int NB>
constexpr int one_mx4_lds() {
    constexpr int tiles = (MB + NB) * 32 * kI8Tile, stage = 4 * (MB % 2 == 0 ? 32 : 16) * (NB * 16 * (int)sizeof(TO) + 16);
    return tiles > stage ? tiles : stage;
}

template <typename TO, int MB, int NB>
__global__ __launch_bounds__(256) void gemm_mx4_one_kernel(const GemmMx4Args a) {
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
    f32x4 acc[MB][NB];
#pragma unroll
    for (int mi = 0; mi < MB; ++mi)
#pragma unroll
        for (int ni = 0; ni < NB; ++ni) acc[mi][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
    uint32_t sx[MB], sw[NB];
    {
        const auto rx = ScaleRows(a.q_scale, a.T, row0, rows, a.d_in).chunk(0);
        const auto rw = ScaleRows(a.w_scale + (size_t)e * mx4_scale_bytes(a.d_out, a.d_in * 2), a.d_out, n0, cols, a.d_in).chunk(0);
#pragma unroll
        for (int i = 0; i < MB; ++i) sx[i] = __builtin_amdgcn_raw_buffer_load_b32(rx, (uint32_t)(wm + i * 16 + l15) * 16 + kq * 4, 0, 0);
#pragma unroll
        for (int i = 0; i < NB; ++i) sw[i] = __builtin_amdgcn_raw_buffer_load_b32(rw, (uint32_t)(wn + i * 16 + l15) * 16 + kq * 4, 0, 0);
    }
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
                acc[mi][ni] = ks == 0 ? mfma_mx4<0>(__builtin_bit_cast(u32x4, f.w[ni]), __builtin_bit_cast(u32x4, f.x[mi]), acc[mi][ni], sw[ni], sx[mi])
                                      : mfma_mx4<1>(__builtin_bit_cast(u32x4, f.w[ni]), __builtin_bit_cast(u32x4, f.x[mi]), acc[mi][ni], sw[ni], sx[mi]);
    }
    ring_mx4_epilogue<TO, MB, NB, true>(a, acc, smem, e, row0, rows, n0, wm, wn, wave, lane);
}

template <typename TO, int TB, int RB, int WV, int D>
static hipError_t launch_wave(GemmMx4Args a, hipStream_t stream) {
    a.tiles_m = most_row_tiles(a, TB * 16);
    a.tile_cols = wave_tile_cols(a.tiles_m, a.d_out, RB * 16);
    a.tiles_n = ceil_div(a.d_out, a.tile_cols);
    constexpr int lds = wave_mx4_lds<TB, RB, WV, D>();
    const auto kern = &gemm_mx4_wave_kernel<TO, TB, RB, WV, D>;
    static_assert(lds <= 160 * 1024, "LDS");
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(kern), lds);
    if (e != hipSuccess) return e;
    if ((int64_t)a.tiles_m * a.tiles_n * WV * 64 >= (int64_t)1 << 32) return hipErrorInvalidValue;
    kern<<<a.tiles_m * a.tiles_n, WV * 64, lds, stream>>>(a);
    return hipGetLastError();
}

template <typename TO, int MB, int NB, int D>
static hipError_t launch_ring_mx4(GemmMx4Args a, hipStream_t stream) {
    a.tiles_m = most_row_tiles(a, MB * 32);
    a.tiles_n = ceil_div(a.d_out, NB * 32);
    constexpr int lds = ring_mx4_lds<MB, NB, D>();
    const auto kern = a.d_in % kI8Tile != 0 ? &gemm_mx4_ring_kernel<TO, MB, NB, D, true> : &gemm_mx4_ring_kernel<TO, MB, NB, D, false>;
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(kern), lds);
    if (e != hipSuccess) return e;
    if ((int64_t)a.tiles_m * a.tiles_n * 256 >= (int64_t)1 << 32) return hipErrorInvalidValue;
    kern<<<a.tiles_m * a.tiles_n, 256, lds, stream>>>(a);
    return hipGetLastError();
}

template <typename TO>
static hipError_t launch_largest_mx4(GemmMx4Args a, hipStream_t stream) {
    const int64_t tiles = (int64_t)most_row_tiles(a, 256) * ceil_div(a.d_out, 256);
    a.tail = may_have_tail(a, tiles) ? 1 : 0;
    const hipError_t e = launch_ring_mx4<TO, 8, 8, 2>(a, stream);
    if (e != hipSuccess || a.tail == 0) return e;
    a.tiles_m = most_row_tiles(a, 256);
    a.tiles_n = ceil_div(a.d_out, 256);
    const auto kern = a.d_in % kI8Tile != 0 ? &gemm_mx4_tail_kernel<TO, true> : &gemm_mx4_tail_kernel<TO, false>;
    const hipError_t f = ensure_lds_limit(reinterpret_cast<const void*>(kern), tail_mx4_lds());
    if (f != hipSuccess) return f;
    const int rest = (int)tiles - tail_start((int)tiles);
    const int wgs = a.offsets != nullptr ? kTailTiles * 4 : rest <= kTailSmall ? rest * 16 : rest <= kTailMiddle ? rest * 8 : rest * 4;
    kern<<<wgs, 256, tail_mx4_lds(), stream>>>(a);
    return hipGetLastError();
}

template <typename TO, int MB, int NB>
static hipError_t launch_one_mx4(GemmMx4Args a, hipStream_t stream) {
    static_assert(MB >= 2, "order of the fragments");
    a.tiles_m = most_row_tiles(a, MB * 32);
    a.tiles_n = ceil_div(a.d_out, NB * 32);
    constexpr int lds = one_mx4_lds<TO, MB, NB>();
    const auto kern = &gemm_mx4_one_kernel<TO, MB, NB>;
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(kern), lds);
    if (e != hipSuccess) return e;
    if ((int64_t)a.tiles_m * a.tiles_n * 256 >= (int64_t)1 << 32) return hipErrorInvalidValue;
    kern<<<a.tiles_m * a.tiles_n, 256, lds, stream>>>(a);
    return hipGetLastError();
}

// ---- which kernel and tile, as for the products of 8-bit integers (see kI8Shapes): a row's bytes count.  The constants of the tiles of 128 x 128
// and more are fitted to the times of all shapes at 269 sizes (27 numbers of rows from 1 to 8192, 10 matrices of 512 to 14336 inputs and 1024 to
// 14336 channels).  The shape that is taken is 0.3 % slower than the best one on average and at most 15 % (512 x 4096 -> 1024, 10.5 and 9.1 us).  300 x
// 4096 -> 4096: 64 x 64 13.7 us, 96 x 64 8.8, 128 x 128 11.4; 2048 x 1024 -> 4096: 128 x 128 two to a CU 8.8, 256 x 256 12.2; 1024 x 4096 -> 14336:
// 128 x 128 42.3, 256 x 128 39.3, 256 x 256 31.9; 8192 x 4096 -> 14336: 330, 271, 227 (4.2 PFLOP/s).
constexpr I8Shape kMx4Shapes[kI8ShapeCount] = {
    {16, 16, 1, true, 2.92f, 1.00f, 0.039f, 0.017f},
    {16, 32, 1, true, 1.31f, 2.84f, 0.036f, 0.060f},
    {16, 64, 1, true, 0.41f, 3.85f, 0.088f, 0.052f},
    {32, 32, 1, true, 1.80f, 2.49f, 0.049f, 0.077f},
    {64, 64, 1, false, 1.00f, 3.07f, 0.145f, 0.110f},
    {96, 64, 1, false, 1.07f, 3.08f, 0.185f, 0.108f},
    {128, 64, 1, false, 1.07f, 3.12f, 0.229f, 0.102f},
    {128, 128, 1, false, 1.13f, 2.81f, 0.474f, 0.104f},
    {128, 128, 2, false, 1.29f, 2.81f, 0.480f, 0.328f},
    {192, 128, 1, false, 0.98f, 4.04f, 0.589f, 0.177f},
    {224, 128, 1, false, 0.91f, 3.47f, 0.650f, 0.178f},
    {256, 128, 1, false, 0.78f, 4.19f, 0.681f, 0.239f},
    {256, 256, 1, false, 0.84f, 6.34f, 0.853f, 0.700f},
};
template <typename TO>
static hipError_t launch_mx4(const GemmMx4Args& a, hipStream_t stream) {
    if (a.d_in <= kI8Tile) return launch_one_mx4<TO, 2, 4>(a, stream);
    switch (choose_shape(a, kMx4Shapes)) {
        case 0: return launch_wave<TO, 1, 1, 4, 5>(a, stream);
        case 1: return launch_wave<TO, 1, 2, 4, 5>(a, stream);
        case 2: return launch_wave<TO, 1, 4, 4, 3>(a, stream);
        case 3: return launch_wave<TO, 2, 2, 4, 4>(a, stream);
        case 4: return launch_ring_mx4<TO, 2, 2, 5>(a, stream);
        case 5: return launch_ring_mx4<TO, 3, 2, 5>(a, stream);
        case 6: return launch_ring_mx4<TO, 4, 2, 4>(a, stream);
        case 7: return launch_ring_mx4<TO, 4, 4, 3>(a, stream);
        case 8: return launch_ring_mx4<TO, 4, 4, 2>(a, stream);
        case 9: return launch_ring_mx4<TO, 6, 4, 3>(a, stream);
        case 10: return launch_ring_mx4<TO, 7, 4, 2>(a, stream);
        case 11: return launch_ring_mx4<TO, 8, 4, 2>(a, stream);
        default: return launch_largest_mx4<TO>(a, stream);
    }
}

template <typename TX, int RB, int D>
static hipError_t launch_row(GemmMx4Args a, const TX* x, hipStream_t stream) {
    a.tile_cols = wave_tile_cols(1, a.d_out, RB * 16);
    a.tiles_n = ceil_div(a.d_out, a.tile_cols);
    const int lds = row_mx4_ring_bytes<RB, D>() + row_mx4_bytes(a.T, a.d_in * 2);
    auto go = [&](auto kern) {
        const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(kern), row_mx4_lds_most<RB, D>());
        if (e != hipSuccess) return e;
        kern<<<a.tiles_n, kRowThreads, lds, stream>>>(a, x);
        return hipGetLastError();
    };
    const int held = ceil_div(a.T * mx4_chunks(a.d_in * 2) * kMxChunk, kRowThreads * 8);
    return held <= 2 ? go(&gemm_mx4_row_kernel<TX, RB, D, 2>) : held <= 9 ? go(&gemm_mx4_row_kernel<TX, RB, D, 9>) : go(&gemm_mx4_row_kernel<TX, RB, D, kRowHeld>);
}
bool base_gemm_mx4_in_one(int T, int d_in, int d_out) {
    return T <= kRowMaxTokens && T * mx4_chunks(d_in) * kMxChunk <= (d_out <= 4096 ? kRowMaxInputs : d_out <= 8192 ? 20480 : 12288);
}

template <typename TX>
static hipError_t launch_base(const GemmMx4Args& a, const TX* x, hipStream_t stream) {
    return a.d_out <= 4096 ? launch_row<TX, 1, 5>(a, x, stream) : launch_row<TX, 2, 4>(a, x, stream);
}
hipError_t launch_base_gemm_mx4_in_one(const void* x, const uint8_t* W, const uint8_t* w_scale, int T, int d_in, int d_out, bool bf16, void* out,
                                       hipStream_t stream) {
    const GemmMx4Args a{nullptr, nullptr, (const int8_t*)W, w_scale, nullptr, out, T, d_in / 2, d_out, 1, 1, 0, 0, 0, 0};
    return bf16 ? launch_base(a, (const bf16_t*)x, stream) : launch_base(a, (const float*)x, stream);
}

static GemmMx4Args mx4_args(const uint8_t* q, const uint8_t* q_scale, const uint8_t* W, const uint8_t* w_scale, const int32_t* offsets,
                            int T, int d_in, int d_out, int N, void* out) {
    const int past_caches = (int64_t)N * d_out * (d_in / 2) >= 100000000;
    return {(const int8_t*)q, q_scale, (const int8_t*)W, w_scale, offsets, out, T, d_in / 2, d_out, N, 0, 0, 0, 0, past_caches};
}
hipError_t launch_gemm_mx4(const uint8_t* q, const uint8_t* q_scale, const uint8_t* W, const uint8_t* w_scale, const int32_t* offsets,
                           int T, int d_in, int d_out, int N, bool bf16, void* out, hipStream_t stream) {
    const GemmMx4Args a = mx4_args(q, q_scale, W, w_scale, offsets, T, d_in, d_out, N, out);
    return bf16 ? launch_mx4<bf16_t>(a, stream) : launch_mx4<float>(a, stream);
}

I8Plan gemm_mx4_plan(int T, int d_in, int d_out, int N, bool grouped) {
    static const int32_t some = 0;   // offsets, which the host does not read
    const GemmMx4Args a = mx4_args(nullptr, nullptr, nullptr, nullptr, grouped ? &some : nullptr, T, d_in, d_out, N, nullptr);
    if (a.d_in <= kI8Tile) return {"one", 64, 128, 1, false, false};
    const I8Shape& s = kMx4Shapes[choose_shape(a, kMx4Shapes)];
    const bool largest = s.rows * s.cols == 256 * 256;
    return {s.wave ? "wave" : "ring", s.rows, s.cols, s.per_cu, !s.wave && !largest && a.past_caches != 0,
            largest && may_have_tail(a, (int64_t)most_row_tiles(a, 256) * ceil_div(d_out, 256))};
}

template <typename TO, int TB, int RB, int WV, int D>
static hipError_t init_wave() {
    return ensure_lds_limit(reinterpret_cast<const void*>(&gemm_mx4_wave_kernel<TO, TB, RB, WV, D>), wave_mx4_lds<TB, RB, WV, D>());
}
template <typename TO, int MB, int NB, int D>
static hipError_t init_ring() {
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(&gemm_mx4_ring_kernel<TO, MB, NB, D, true>), ring_mx4_lds<MB, NB, D>());
    return e != hipSuccess ? e : ensure_lds_limit(reinterpret_cast<const void*>(&gemm_mx4_ring_kernel<TO, MB, NB, D, false>), ring_mx4_lds<MB, NB, D>());
}
template <typename TO>
static hipError_t init_tail() {
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(&gemm_mx4_tail_kernel<TO, true>), tail_mx4_lds());
    return e != hipSuccess ? e : ensure_lds_limit(reinterpret_cast<const void*>(&gemm_mx4_tail_kernel<TO, false>), tail_mx4_lds());
}
template <typename TX, int RB, int D>
static hipError_t init_row() {
    hipError_t e = hipSuccess;
    for (const void* k : {reinterpret_cast<const void*>(&gemm_mx4_row_kernel<TX, RB, D, 2>), reinterpret_cast<const void*>(&gemm_mx4_row_kernel<TX, RB, D, 9>),
                          reinterpret_cast<const void*>(&gemm_mx4_row_kernel<TX, RB, D, kRowHeld>)})
        if (e == hipSuccess) e = ensure_lds_limit(k, row_mx4_lds_most<RB, D>());
    return e;
}
template <typename TO>
static hipError_t init_mx4() {   // every kernel that launch_mx4 and launch_base may start
    hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(&gemm_mx4_one_kernel<TO, 2, 4>), one_mx4_lds<TO, 2, 4>());
    for (hipError_t f : {init_wave<TO, 1, 1, 4, 5>(), init_wave<TO, 1, 2, 4, 5>(), init_wave<TO, 1, 4, 4, 3>(), init_wave<TO, 2, 2, 4, 4>(),
                         init_ring<TO, 2, 2, 5>(), init_ring<TO, 3, 2, 5>(), init_ring<TO, 4, 2, 4>(), init_ring<TO, 4, 4, 3>(),
                         init_ring<TO, 4, 4, 2>(), init_ring<TO, 6, 4, 3>(), init_ring<TO, 7, 4, 2>(), init_ring<TO, 8, 4, 2>(),
                         init_ring<TO, 8, 8, 2>(), init_tail<TO>(), init_row<TO, 1, 5>(), init_row<TO, 2, 4>()})
        if (e == hipSuccess) e = f;
    return e;
}
hipError_t gemm_mx4_init_kernels() {
    const hipError_t e = init_mx4<bf16_t>();
    return e != hipSuccess ? e : init_mx4<float>();
}

}  // namespace meteora
