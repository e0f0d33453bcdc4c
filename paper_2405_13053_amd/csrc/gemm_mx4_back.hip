// Gradient of a projection with its weight in 4 bits (quant_mx4.hpp) with respect to a few tokens' rows, from the codes themselves:
//
//     dx[t,i] = sum_o dy[t,o] * 2^(E[o, i / 32] - 127) * W[o,i]
//
// The sum runs over rows of W, whose neighbours in memory are values of other sums, and every row has a scale of its own.  So a lane takes 8 inputs of 8
// consecutive rows, makes them bf16, exactly, and turns them in registers: a perm to two values, after which 4 registers are 8 consecutive
// terms of one input's sum, a lane's part of the first operand of v_mfma_f32_16x16x32_bf16.  The 16 rows of that operand are inputs 8 apart,
// one of each lane's, and its 8 instructions to 16 tokens together give every lane 8 consecutive inputs of a token.
//
// A workgroup has 128 inputs and up to 64 tokens; its 8 wavefronts, and `splits` workgroups, share out the rows of W, 32 to a step.  A wavefront's steps
// come through a ring of its own in LDS: 64 bytes of each row, its 16 bytes of scales, and 32 columns of dy.  The wavefronts' sums are added
// in LDS, the workgroups' by a second launch, in one order.
#include "common.hpp"
#include "gemm_mfma.hpp"
#include "gemm_rows.hpp"
#include "kernels.hpp"
#include "quant_mx4.hpp"

namespace meteora {

constexpr int kBackWaves = 8, kBackInputs = 128, kBackStep = 32, kBackTokens = 64;
constexpr int kBackSum = 8 * (1024 + 16);   // bytes of a wavefront's sums of 16 tokens: 8 registers of 4 values; 4 banks apart

struct MxBackArgs {
    const bf16_t* dy;        // [T, d_out]
    const uint8_t *W, *scale;
    bf16_t* dx;              // [T, d_in], without splits
    float* part;             // [splits][T, d_in], or nullptr
    int T, d_in, d_out, tiles, blocks, splits;   // of 128 inputs, of 64 tokens
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t back_rsrc(const void* p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}

__device__ __forceinline__ void back_load(__amdgpu_buffer_rsrc_t from, unsigned char* to, uint32_t at) {   // 16 bytes to each lane
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, at, 0, 0, 0);
}
__device__ __forceinline__ f32x4 back_mfma(const bf16x8& w, const bf16x8& x, const f32x4& acc) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, acc, 0, 0, 0);
}

template <int TB> constexpr int back_slot() { return 2048 + 1024 + TB * 1024; }
template <int TB> constexpr int kBackDepth = TB == 1 ? 4 : TB == 2 ? 3 : 2;
template <int TB>
constexpr int back_lds() {
    constexpr int ring = kBackWaves * kBackDepth<TB> * back_slot<TB>(), sums = kBackWaves * (TB < 2 ? TB : 2) * kBackSum;
    return ring > sums ? ring : sums;
}
static_assert(back_lds<1>() <= 160 * 1024 && back_lds<2>() <= 160 * 1024 && back_lds<4>() <= 160 * 1024, "LDS");

// Offsets stay in 31 bits: 64 rows of dy are 128 MB at most, 32 of W 2 MB.  What bounds it is how soon the codes come (1 token of 5120 -> 13824, 38 MB, 14 us
// and 3 for the second launch) and, from 33 tokens on, the matrix instructions: 512 x 4096 -> 4096 0.69 PFLOP/s, 512 x 4096 -> 14336 0.82.
template <int TB>
__global__ __launch_bounds__(kBackWaves * 64) void gemm_mx4_back_kernel(const MxBackArgs a) {
    constexpr int D = kBackDepth<TB>, NL = 3 + TB, kSlot = back_slot<TB>();
    static_assert((D - 1) * NL < 64, "vmcnt");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, kq = lane >> 4;
    const int id = xcd_order(blockIdx.x, a.tiles * a.blocks * a.splits);   // blocks of tokens, then tiles of the same rows next to each other
    const int block = id % a.blocks, rest = id / a.blocks, part = rest / a.tiles, i0 = (rest - part * a.tiles) * kBackInputs;
    const int t0 = block * kBackTokens, tokens = min(kBackTokens, a.T - t0);
    const int all = ceil_div(a.d_out, kBackStep), share = ceil_div(all, a.splits), end = min(all, part * share + share);
    const uint32_t bytes = (uint32_t)a.d_in / 2, ld = (uint32_t)a.d_out * 2;

    // Row kq * 8 + r of a step lies at position r * 4 + kq, so that a read of the four kq's is one piece of LDS
    const auto row_at = [](int p) { return (p & 3) * 8 + (p >> 2); };
    uint32_t at_w[2], at_dy[TB];
    const uint32_t chunk = (uint32_t)i0 / 2 + (lane & 3) * 16;   // d_in % 32 == 0: there or not
#pragma unroll
    for (int j = 0; j < 2; ++j) at_w[j] = chunk < bytes ? (uint32_t)row_at(j * 16 + (lane >> 2)) * bytes + chunk : kOutside;
    const uint32_t at_s = lane < kBackStep ? (uint32_t)row_at(lane) * 16 : kOutside;
#pragma unroll
    for (int b = 0; b < TB; ++b) {
        const int t = b * 16 + (lane >> 2);
        at_dy[b] = t < tokens ? (uint32_t)t * ld + (lane & 3) * 16 : kOutside;
    }
    const auto dy = back_rsrc(a.dy + (size_t)t0 * a.d_out, (uint32_t)tokens * ld);
    const uint8_t* const scale = a.scale + (size_t)(i0 / kMxChunk) * ((size_t)a.d_out * 16);
    unsigned char* const ring = smem + wave * D * kSlot;
    int req = part * share + wave, req_at = 0;
    const auto request = [&] {   // behind the last step: of no rows
        unsigned char* const slot = ring + req_at * kSlot;
        req_at = req_at + 1 == D ? 0 : req_at + 1;
        const int o = req * kBackStep, rows = req < end ? min(kBackStep, a.d_out - o) : 0;
        const auto w = back_rsrc(a.W + (size_t)o * bytes, (uint32_t)rows * bytes);
        const auto s = back_rsrc(scale + (size_t)o * 16, (uint32_t)rows * 16);
#pragma unroll
        for (int j = 0; j < 2; ++j)
            back_load(w, slot + j * 1024, at_w[j]);
        back_load(s, slot + 2048, at_s);
        const bool there = (lane & 3) * 8 < rows;   // columns of dy; d_out % 8 == 0
#pragma unroll
        for (int b = 0; b < TB; ++b)
            back_load(dy, slot + 3072 + b * 1024, there && at_dy[b] != kOutside ? at_dy[b] + (uint32_t)o * 2 : kOutside);
        req += kBackWaves;
    };
#pragma unroll
    for (int i = 0; i < D; ++i) request();
    f32x4 acc[8][TB];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int b = 0; b < TB; ++b) acc[j][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int quarter = (i0 / kBackInputs & 3) * 8;   // block b of a chunk has byte b / 4 of word b % 4
    int at = 0;
    for (int s = part * share + wave; s < end; s += kBackWaves) {
        const unsigned char* const slot = ring + at * kSlot;
        at = at + 1 == D ? 0 : at + 1;
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * NL) : "memory");
        uint32_t w[8], e[8];
        bf16x8 x[TB];
#pragma unroll
        for (int r = 0; r < 8; ++r) w[r] = *reinterpret_cast<const uint32_t*>(slot + (r * 4 + kq) * 64 + l15 * 4);
#pragma unroll
        for (int r = 0; r < 8; ++r) e[r] = *reinterpret_cast<const uint32_t*>(slot + 2048 + (r * 4 + kq) * 16 + (l15 >> 2) * 4);
#pragma unroll
        for (int b = 0; b < TB; ++b) x[b] = *reinterpret_cast<const bf16x8*>(slot + 3072 + b * 1024 + (l15 * 4 + kq) * 16);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slot is read
        request();
        u32x4 v[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] = mx4_bf16x8(w[r], mx4_scale(e[r] >> quarter & 255));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            u32x4 f;
#pragma unroll
            for (int k = 0; k < 4; ++k) f[k] = __builtin_amdgcn_perm(v[2 * k + 1][j >> 1], v[2 * k][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int b = 0; b < TB; ++b) acc[j][b] = back_mfma(__builtin_bit_cast(bf16x8, f), x[b], acc[j][b]);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may land in what follows
    // 16 or 32 tokens at a time: [wavefront][block][j][lane], added by a thread for two neighbouring inputs of four pieces of 8
    constexpr int B = TB < 2 ? TB : 2;
    const int jq = tid & 3, from = tid >> 2 & 63, mine = tid >> 8;
#pragma unroll
    for (int b0 = 0; b0 < TB; b0 += B) {
        __syncthreads();
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
            for (int j = 0; j < 8; ++j) *reinterpret_cast<f32x4*>(smem + (wave * B + b) * kBackSum + j * 1040 + lane * 16) = acc[j][b0 + b];
        __syncthreads();
        const int t = (b0 + mine) * 16 + (from & 15);
        if (mine < B && t < tokens) {
            f32x4 sum[2] = {};
#pragma unroll
            for (int v = 0; v < kBackWaves; ++v)
#pragma unroll
                for (int h = 0; h < 2; ++h) sum[h] += *reinterpret_cast<const f32x4*>(smem + (v * B + mine) * kBackSum + (jq * 2 + h) * 1040 + from * 16);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int i = i0 + ((from >> 4) * 4 + c) * 8 + jq * 2;
                const size_t o = (size_t)(t0 + t) * a.d_in + i;
                if (i < a.d_in) {
                    if (a.part != nullptr) *reinterpret_cast<float2*>(a.part + (size_t)part * a.T * a.d_in + o) = make_float2(sum[0][c], sum[1][c]);
                    else *reinterpret_cast<uint32_t*>(a.dx + o) = pack_bf16x2(sum[0][c], sum[1][c]);
                }
            }
        }
    }
}

__global__ __launch_bounds__(256) void gemm_mx4_back_sum_kernel(const float* __restrict__ part, int splits, size_t all, bf16_t* __restrict__ dx) {
    const size_t o = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (o >= all) return;
    f32x4 sum = *reinterpret_cast<const f32x4*>(part + o);
    for (int p = 1; p < splits; ++p) sum += *reinterpret_cast<const f32x4*>(part + (size_t)p * all + o);
    *reinterpret_cast<uint2*>(dx + o) = make_uint2(pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3]));
}

// Or dequantize_mx4_turned_kernel and a product of bf16 matrices, which reads W's 16 bits a value again, in tiles of more tokens.  From the codes and so, us:
// 4096 -> 4096, 1, 32, 64, 256 and 512 tokens 10.1, 12.4, 16.7, 19.9, 24.9 and 30.6, 29.9, 31.1, 29.2, 33.1; 5120 -> 13824 17.9, 20.2, 25.1, 66.7, 125
// and 62.9, 63.5, 65.6, 79.4, 110; 14336 -> 4096, 256 and 512, 448 and 896 workgroups, 48.9 and 93.0, and 59.5 and 75.6; 4096 -> 14336, 512, 256
// workgroups, 73.5 and 92.6; 2048 -> 8192, 1024 and 1536 42.2 and 79.4, and 47.5 and 57.8.
bool mx4_back_takes(int T, int d_in) {
    return T <= 256 || (T <= 1024 && ceil_div(d_in, kBackInputs) * ceil_div(T, kBackTokens) <= 256);
}
// Workgroups to a tile: as fill the CUs once, with a step to every wavefront, as far as there is room for their sums
static int back_splits(int T, int d_in, int d_out, size_t room) {
    const int tiles = ceil_div(d_in, kBackInputs) * ceil_div(T, kBackTokens), steps = ceil_div(d_out, kBackStep);
    int n = tiles < 256 ? 256 / tiles : 1;
    n = n < steps / kBackWaves ? n : steps / kBackWaves;
    const size_t fit = room / ((size_t)T * d_in * sizeof(float));
    n = (size_t)n < fit ? n : (int)fit;
    return n < 1 ? 1 : ceil_div(steps, ceil_div(steps, n));   // none without steps
}
template <int TB>
static hipError_t launch_back(const MxBackArgs& a, hipStream_t stream) {
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(&gemm_mx4_back_kernel<TB>), back_lds<TB>());
    if (e != hipSuccess) return e;
    gemm_mx4_back_kernel<TB><<<a.tiles * a.blocks * a.splits, kBackWaves * 64, back_lds<TB>(), stream>>>(a);
    return hipGetLastError();
}
hipError_t launch_mx4_back(const void* dy, const uint8_t* W, const uint8_t* scale, int T, int d_in, int d_out, void* dx, void* ws, size_t room,
                           hipStream_t stream) {
    const int splits = back_splits(T, d_in, d_out, room);
    const MxBackArgs a{(const bf16_t*)dy, W, scale, (bf16_t*)dx, splits > 1 ? (float*)ws : nullptr, T, d_in, d_out, ceil_div(d_in, kBackInputs),
                       ceil_div(T, kBackTokens), splits};
    const hipError_t e = T <= 16 ? launch_back<1>(a, stream) : T <= 32 ? launch_back<2>(a, stream) : launch_back<4>(a, stream);
    if (e != hipSuccess || splits == 1) return e;
    const size_t all = (size_t)T * d_in;
    gemm_mx4_back_sum_kernel<<<(int)((all + 1023) / 1024), 256, 0, stream>>>(a.part, splits, all, a.dx);
    return hipGetLastError();
}
hipError_t mx4_back_init_kernels() {
    hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(&gemm_mx4_back_kernel<1>), back_lds<1>());
    if (e == hipSuccess) e = ensure_lds_limit(reinterpret_cast<const void*>(&gemm_mx4_back_kernel<2>), back_lds<2>());
    if (e == hipSuccess) e = ensure_lds_limit(reinterpret_cast<const void*>(&gemm_mx4_back_kernel<4>), back_lds<4>());
    return e;
}

}  // namespace meteora
