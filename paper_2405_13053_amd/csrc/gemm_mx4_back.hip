// Gradient of a projection with its weight in 4 bits (quant_mx4.hpp) with respect to its input from the codes themselves, for some hundred tokens in bf16 and for
// most batches in fp32 (see mx4_back_takes):
//
//     dx[t,i] = sum_o dy[t,o] * 2^(E[o, i / 32] - 127) * W[o,i]
//
// The sum runs over rows of W, whose neighbours in memory are values of other sums, and every row has a scale of its own.  So a lane takes 8 inputs of 8
// consecutive rows, makes them bf16, exactly, and turns them in registers: a perm to two values, after which 4 registers are 8 consecutive
// terms of one input's sum, a lane's part of the first operand of v_mfma_f32_16x16x32_bf16.  The 16 rows of that operand are inputs 8 apart,
// one of each lane's, and its 8 instructions to 16 tokens together give every lane 8 consecutive inputs of a token.
//
// A workgroup has 128 inputs and up to 64 tokens (fp32: 32); its 8 wavefronts, and `splits` workgroups, share out the rows of W, 32 to a step.  A wavefront's steps
// come through a ring of its own in LDS: 64 bytes of each row, its 16 bytes of scales, and 32 columns of dy.  The wavefronts' sums are added
// in LDS, the workgroups' by a second launch, in one order.
#include "common.hpp"
#include "gemm_mfma.hpp"
#include "gemm_rows.hpp"
#include "kernels.hpp"
#include "quant_mx4.hpp"

namespace meteora {

constexpr int kBackWaves = 8, kBackInputs = 128, kBackStep = 32;
template <typename TX> constexpr int kBackTokens = sizeof(TX) == 2 ? 64 : 32;   // of a workgroup
constexpr int kBackScales = kBackStep * kBackInputs / 2, kBackDy = kBackScales + 1024;   // where scales (of 32 rows; room for 64 pieces) and dy are in a slot
constexpr int kBackSum = 8 * (1024 + 16);   // bytes of a wavefront's sums of 16 tokens: 8 registers of 4 values; 4 banks apart

struct MxBackArgs {
    const void* dy;          // [T, d_out]
    const uint8_t *W, *scale;
    void* dx;                // [T, d_in], without splits
    float* part;             // [splits][T, d_in], or nullptr
    int T, d_in, d_out, tiles, blocks, splits;   // of 128 inputs, of kBackTokens tokens
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

template <typename TX, int TB> constexpr int back_slot() { return kBackDy + TB * 512 * (int)sizeof(TX); }
template <typename TX, int TB> constexpr int kBackDepth = back_slot<TX, TB>() <= 4096 ? 4 : back_slot<TX, TB>() <= 5120 ? 3 : 2;
template <typename TX, int TB>
constexpr int back_lds() {
    constexpr int ring = kBackWaves * kBackDepth<TX, TB> * back_slot<TX, TB>(), sums = kBackWaves * (TB < 2 ? TB : 2) * kBackSum;
    return ring > sums ? ring : sums;
}
static_assert(back_lds<bf16_t, 1>() <= 160 * 1024 && back_lds<bf16_t, 2>() <= 160 * 1024 && back_lds<bf16_t, 4>() <= 160 * 1024, "LDS");
static_assert(back_lds<float, 1>() <= 160 * 1024 && back_lds<float, 2>() <= 160 * 1024, "LDS");

// 8 columns of a token as operands: a bf16 number is one, an fp32 number the sum of three, its first 8 bits, the next 8 and the last.  Products with W's two
// bits are exact, so that the sum is as good as one of fp32 products, at a third of the bf16 rate, five times that of fp32.  What is no number stays
// in the first; the parts of one under 2^-110 may be lost under the least bf16 number.
template <typename TX> constexpr int kBackParts = sizeof(TX) == 2 ? 1 : 3;
__device__ __forceinline__ void back_parts(const unsigned char* tokens, int l15, int kq, bf16x8 (&x)[1]) {
    x[0] = *reinterpret_cast<const bf16x8*>(tokens + (l15 * 4 + kq) * 16);
}
__device__ __forceinline__ void back_parts(const unsigned char* tokens, int l15, int kq, bf16x8 (&x)[3]) {   // 16-byte piece c of row t is at c ^ t % 8
    u32x4 part[3];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(tokens + l15 * 128 + ((kq * 2 + h) ^ (l15 & 7)) * 16);
        uint32_t p[3][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u = v[i], size = u & 0x7fffffffu;
            const bool number = size < 0x7f800000u;
            p[0][i] = size > 0x7f800000u ? u | 0x00400000u : u;
            const float rest = number ? __uint_as_float(u) - __uint_as_float(u & 0xffff0000u) : 0.f;
            p[1][i] = __float_as_uint(rest);
            p[2][i] = __float_as_uint(rest - __uint_as_float(p[1][i] & 0xffff0000u));
        }
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) part[k][h * 2 + i] = __builtin_amdgcn_perm(p[k][2 * i + 1], p[k][2 * i], 0x07060302u);   // the upper halves
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) x[k] = __builtin_bit_cast(bf16x8, part[k]);
}
__device__ __forceinline__ void back_store(bf16_t* to, float a, float b) { *reinterpret_cast<uint32_t*>(to) = pack_bf16x2(a, b); }
__device__ __forceinline__ void back_store(float* to, float a, float b) { *reinterpret_cast<float2*>(to) = make_float2(a, b); }

// Offsets stay in 31 bits: 64 rows of dy are 128 MB at most, 32 of W 2 MB.  What bounds it is how soon the codes come (1 token of 5120 -> 13824, 38 MB, 14 us
// and 3 for the second launch) and, from 33 tokens on, the matrix instructions: 512 x 4096 -> 4096 0.69 PFLOP/s, 512 x 4096 -> 14336 0.82.
template <typename TX, int TB>
__global__ __launch_bounds__(kBackWaves * 64) void gemm_mx4_back_kernel(const MxBackArgs a) {
    constexpr int D = kBackDepth<TX, TB>, EB = sizeof(TX), kSlot = back_slot<TX, TB>();
    constexpr int PER = EB * 2, ROWS = 64 / PER, ND = TB * 16 / ROWS, NL = 3 + ND, P = kBackParts<TX>;   // 16-byte pieces of a token, tokens of a load instruction
    static_assert((D - 1) * NL < 64, "vmcnt");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, kq = lane >> 4;
    const int id = xcd_order(blockIdx.x, a.tiles * a.blocks * a.splits);   // blocks of tokens, then tiles of the same rows next to each other
    const int block = id % a.blocks, rest = id / a.blocks, part = rest / a.tiles, i0 = (rest - part * a.tiles) * kBackInputs;
    const int t0 = block * kBackTokens<TX>, tokens = min(kBackTokens<TX>, a.T - t0);
    const int all = ceil_div(a.d_out, kBackStep), share = ceil_div(all, a.splits), end = min(all, part * share + share);
    const uint32_t bytes = (uint32_t)a.d_in / 2, ld = (uint32_t)a.d_out * EB;

    // Row kq * 8 + r of a step lies at position r * 4 + kq, so that a read of the four kq's is one piece of LDS
    const auto row_at = [](int p) { return (p & 3) * 8 + (p >> 2); };
    uint32_t at_w[2], at_dy[ND];
    const uint32_t chunk = (uint32_t)i0 / 2 + (lane & 3) * 16;   // d_in % 32 == 0: there or not
#pragma unroll
    for (int j = 0; j < 2; ++j) at_w[j] = chunk < bytes ? (uint32_t)row_at(j * 16 + (lane >> 2)) * bytes + chunk : kOutside;
    const int piece = EB == 2 ? lane & 3 : (lane & 7) ^ (lane >> 3);   // of dy, see back_parts
    const uint32_t at_s = lane < kBackStep ? (uint32_t)row_at(lane) * 16 : kOutside;
#pragma unroll
    for (int b = 0; b < ND; ++b) {
        const int t = b * ROWS + lane / PER;
        at_dy[b] = t < tokens ? (uint32_t)t * ld + piece * 16 : kOutside;
    }
    const auto dy = back_rsrc(static_cast<const TX*>(a.dy) + (size_t)t0 * a.d_out, (uint32_t)tokens * ld);
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
        back_load(s, slot + kBackScales, at_s);
        const bool there = piece * (16 / EB) < rows;   // columns of dy; d_out % 8 == 0
#pragma unroll
        for (int b = 0; b < ND; ++b)
            back_load(dy, slot + kBackDy + b * 1024, there && at_dy[b] != kOutside ? at_dy[b] + (uint32_t)o * EB : kOutside);
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
        bf16x8 x[TB][P];
#pragma unroll
        for (int r = 0; r < 8; ++r) w[r] = *reinterpret_cast<const uint32_t*>(slot + (r * 4 + kq) * 64 + l15 * 4);
#pragma unroll
        for (int r = 0; r < 8; ++r) e[r] = *reinterpret_cast<const uint32_t*>(slot + kBackScales + (r * 4 + kq) * 16 + (l15 >> 2) * 4);
#pragma unroll
        for (int b = 0; b < TB; ++b) back_parts(slot + kBackDy + b * 512 * EB, l15, kq, x[b]);
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
            for (int k = P - 1; k >= 0; --k)   // the smallest first
#pragma unroll
                for (int b = 0; b < TB; ++b) acc[j][b] = back_mfma(__builtin_bit_cast(bf16x8, f), x[b][k], acc[j][b]);
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
                    if (a.part != nullptr) back_store(a.part + (size_t)part * a.T * a.d_in + o, sum[0][c], sum[1][c]);
                    else back_store(static_cast<TX*>(a.dx) + o, sum[0][c], sum[1][c]);
                }
            }
        }
    }
}

template <typename TX>
__global__ __launch_bounds__(256) void gemm_mx4_back_sum_kernel(const float* __restrict__ part, int splits, size_t all, TX* __restrict__ dx) {
    const size_t o = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (o >= all) return;
    f32x4 sum = *reinterpret_cast<const f32x4*>(part + o);
#pragma unroll 8
    for (int p = 1; p < splits; ++p) sum += *reinterpret_cast<const f32x4*>(part + (size_t)p * all + o);
    back_store(dx + o, sum[0], sum[1]);
    back_store(dx + o + 2, sum[2], sum[3]);
}

// Or dequantize_mx4_turned_kernel and a product of bf16 matrices, which reads W's 16 bits a value again, in tiles of more tokens.  From the codes and so, us:
// 4096 -> 4096, 1, 32, 64, 256 and 512 tokens 10.1, 12.4, 16.7, 19.9, 24.9 and 30.6, 29.9, 31.1, 29.2, 33.1; 5120 -> 13824 18.2, 22.2, 25.2, 60.6, 125
// and 62.9, 63.5, 65.6, 79.4, 110; 14336 -> 4096, 256 and 512, 448 and 896 workgroups, 48.9 and 93.0, and 59.5 and 75.6; 4096 -> 14336, 512, 256
// workgroups, 73.5 and 92.6; 2048 -> 8192, 1024 and 1536 42.2 and 79.4, and 47.5 and 57.8.  fp32, with products of fp32 matrices: 4096 -> 4096, 1, 64, 512
// and 2048 12.3, 19.4, 71.2 and 272, and 43.6, 79.2, 285 and 703; 5120 -> 13824 19.8, 42.4, 268 and 1045, and 213, 321, 1325 and 3824; 131072 x 4096 ->
// 256 2611 and 3023.  Of few outputs a workgroup has little more than its start and end: 65536 x 4096 -> 8, 64, 128 and 160 989, 996, 1007 and 1176, and 237,
// 510, 843 and 1032, 8192 x 512 -> 8, 96, 128 and 160 21.8, 21.6, 21.7 and 24.4, and 12.8, 21.4, 25.2 and 28.6; that takes more than two rounds of
// workgroups to matter: 2048 x 512 -> 8 7.9 and 9.9, 512 x 4096 -> 8 and 64 12.5 and 12.7, and 12.1 and 16.2.
bool mx4_back_takes(int T, int d_in, int d_out, bool bf16) {
    const int tiles = ceil_div(d_in, kBackInputs);
    if (!bf16) return d_out > kMxBackFewOutputs || (int64_t)tiles * ceil_div(T, kBackTokens<float>) <= 512;
    return T <= 256 || (T <= 1024 && tiles * ceil_div(T, kBackTokens<bf16_t>) <= 256);
}
// Workgroups to a tile: the number that takes the least by rounds of 256 workgroups * (steps of a wavefront * time of one + 3 us), and a second launch and its
// bytes if they are more than one.  A step takes 0.65 to 1.6 us by tokens and type, and 1.0 for all 256 workgroups' codes from memory.  Of 1 token of 512 -> 14336 1,
// 4, 16 and 32 workgroups to a tile take 40.6, 14.8, 10.9 and 11.4 us, of 64 of 4096 -> 1024 1, 2, 4 and 8 10.4, 11.0, 11.7 and 14.1, of 200 of 5120 ->
// 13824, 160 tiles, 1, 3 and 4 62.0, 55.4 and 65.5; over 88 such sizes the choice is 2 % slower than the best.
static int back_splits(int T, int tiles, int d_in, int d_out, bool bf16, size_t room) {
    const int steps = ceil_div(d_out, kBackStep);
    const float one = T <= 16 ? (bf16 ? 0.65f : 1.f) : bf16 ? (T <= 32 ? 0.7f : 0.95f) : 1.6f;
    const size_t sums = (size_t)T * d_in * sizeof(float);
    int best = 1;
    float least = 0.f;
    for (int n = 1; n <= 32 && n <= steps && (n == 1 || sums * n <= room); ++n) {
        const int share = ceil_div(steps, n);
        if (n > 1 && ceil_div(steps, share) != n) continue;   // workgroups without steps
        const int64_t groups = (int64_t)tiles * n;
        const float all = groups < 256 ? (float)groups / 256.f : 1.f, step = one > all ? one : all;
        const float us = (float)((groups + 255) / 256) * ((float)ceil_div(share, kBackWaves) * step + 3.f) + (n > 1 ? 2.f + 0.1f * (float)n + 2.f * (float)sums * (float)n / 5e6f : 0.f);
        if (n == 1 || us < least) { least = us; best = n; }
    }
    return best;
}
template <typename TX, int TB>
static hipError_t launch_tiles(const MxBackArgs& a, hipStream_t stream) {
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(&gemm_mx4_back_kernel<TX, TB>), back_lds<TX, TB>());
    if (e != hipSuccess) return e;
    gemm_mx4_back_kernel<TX, TB><<<a.tiles * a.blocks * a.splits, kBackWaves * 64, back_lds<TX, TB>(), stream>>>(a);
    return hipGetLastError();
}
template <typename TX>
static hipError_t launch_back(MxBackArgs a, size_t room, hipStream_t stream) {
    a.tiles = ceil_div(a.d_in, kBackInputs);
    a.blocks = ceil_div(a.T, kBackTokens<TX>);
    a.splits = back_splits(a.T, a.tiles * a.blocks, a.d_in, a.d_out, sizeof(TX) == 2, room);
    float* const part = a.part;
    if (a.splits == 1) a.part = nullptr;
    hipError_t e;
    if constexpr (sizeof(TX) == 2) e = a.T <= 16 ? launch_tiles<TX, 1>(a, stream) : a.T <= 32 ? launch_tiles<TX, 2>(a, stream) : launch_tiles<TX, 4>(a, stream);
    else e = a.T <= 16 ? launch_tiles<TX, 1>(a, stream) : launch_tiles<TX, 2>(a, stream);
    if (e != hipSuccess || a.splits == 1) return e;
    const size_t all = (size_t)a.T * a.d_in;
    gemm_mx4_back_sum_kernel<<<(int)((all + 1023) / 1024), 256, 0, stream>>>(part, a.splits, all, static_cast<TX*>(a.dx));
    return hipGetLastError();
}
// Batches of up to kBackGroups workgroups, far below the 2^32 threads of a grid; each is 1024 rounds of workgroups, so that their ends cost nothing
constexpr int kBackGroups = 1 << 18;
template <typename TX>
static hipError_t launch_batches(MxBackArgs a, size_t room, hipStream_t stream) {
    const int all = a.T, most = kBackGroups / ceil_div(a.d_in, kBackInputs) * kBackTokens<TX>;   // d_in <= 131072: 1024 tiles at most
    for (int t0 = 0; t0 < all; t0 += most) {
        a.T = all - t0 < most ? all - t0 : most;
        const hipError_t e = launch_back<TX>(a, room, stream);
        if (e != hipSuccess) return e;
        a.dy = static_cast<const TX*>(a.dy) + (size_t)a.T * a.d_out;
        a.dx = static_cast<TX*>(a.dx) + (size_t)a.T * a.d_in;
    }
    return hipSuccess;
}
hipError_t launch_mx4_back(const void* dy, const uint8_t* W, const uint8_t* scale, int T, int d_in, int d_out, bool bf16, void* dx, void* ws, size_t room,
                           hipStream_t stream) {
    const MxBackArgs a{dy, W, scale, dx, (float*)ws, T, d_in, d_out, 0, 0, 0};
    return bf16 ? launch_batches<bf16_t>(a, room, stream) : launch_batches<float>(a, room, stream);
}
hipError_t mx4_back_init_kernels() {
    hipError_t e = hipSuccess;
    const auto set = [&](auto kern, int lds) { if (e == hipSuccess) e = ensure_lds_limit(reinterpret_cast<const void*>(kern), lds); };
    set(&gemm_mx4_back_kernel<bf16_t, 1>, back_lds<bf16_t, 1>());
    set(&gemm_mx4_back_kernel<bf16_t, 2>, back_lds<bf16_t, 2>());
    set(&gemm_mx4_back_kernel<bf16_t, 4>, back_lds<bf16_t, 4>());
    set(&gemm_mx4_back_kernel<float, 1>, back_lds<float, 1>());
    set(&gemm_mx4_back_kernel<float, 2>, back_lds<float, 2>());
    return e;
}

}  // namespace meteora
