// Gated MLPs of the experts that a few tokens (T <= 64) are routed to, and the gate in front of them:
//
//     h[t,j]  = silu(W1_e[0:f] x[t]) * (W1_e[f:2f] x[t]),    e = topk_idx[t,j],    silu(g) = g / (1 + exp(-g))
//     out[t]  = base[t] + scale * sum_j topk_w[t,j] * (W2_e h[t,j])
//
// Weights are bf16, or 4-bit values with block scales (quant_mx4.hpp) that become bf16 in registers, exactly, so that both run on
// v_mfma_f32_16x16x32_bf16 with x as it is: W is the first operand, the tokens are the 16 columns of the second.  h is rounded to bf16 once, as
// the operand of the second product; sums are fp32.  That rounding takes the output's error from 0.0017 of the output, which is its own rounding, to 0.0023.  h as two
// bf16 parts would do without it and double the columns of the second product: 32 tokens' K tiles of 4 bits would no longer leave room for three slots in
// LDS, and blocks of 16 tokens instead read W again (64 tokens of 8 experts, both products in such
// blocks, 174 instead of 150 us), which is why it is not done.
//
// The weights of the experts in use are what there is to read, once, and what the time goes into: 2 experts of 4096 and 14336 in 4 bits, 187 MB, take 42 us
// (4.5 TB/s), 8 of them and 64 tokens 154 (4.9).  Every wavefront streams its rows through a ring of its own (see gemm_rows.hpp), K tiles of 128 bytes
// a row.  Which tokens an expert has every workgroup finds out for itself: a lane holds an expert's tokens as the bits of a word.
//
// up to 4 tokens: the tokens are the columns, 16 rows of W the rows.  experts_few_up_kernel, with the gate of a single token in it, and
//   experts_few_down_kernel, where the wavefronts split K and go through the experts in use one after the other, so that the weighted sum is in
//   registers; where there are few channels workgroups split K too, and experts_few_sum_kernel adds.
// more: an expert's tokens are columns, 16 or 32 at a time, read once for the wavefronts of a workgroup, which have rows of W of their
//   own.  experts_many_kernel for either product, experts_sum_kernel for the rows of a token.
// In front of them gate_part_kernel, and beyond kRouteTokens tokens experts_route_kernel.  Sums are added in one order: results repeat.
#include <stddef.h>

#include <type_traits>

#include "common.hpp"
#include "gemm_mfma.hpp"
#include "gemm_rows.hpp"
#include "kernels.hpp"
#include "quant_mx4.hpp"
#include "topk_key.hpp"

namespace meteora {

constexpr int kFewTokens = 4;
constexpr int kRouteTokens = 16;   // up to here every workgroup of the first product routes, beyond it is a launch of its own

// ---- the gate: logits[j] = sum_i x[i] W_gate[i,j] + bias[j], top-k and softmax.  gate_part_kernel: a slice of the rows of W_gate, 16 values to a
// thread, for 4 tokens; part[t][slice][NP], NP = N rounded up to a power of two.  The slices are added where they are needed, by whoever
// needs the routing: a wavefront to a token.
constexpr int kGateSlices = 32, kGateTokens = 4, kGateHeld = 16;
__host__ __device__ constexpr int gate_columns(int N) { return N <= 8 ? 8 : N <= 16 ? 16 : N <= 32 ? 32 : 64; }
__host__ __device__ constexpr int gate_slice_rows(int NP) { return 256 * kGateHeld / NP; }
__host__ __device__ constexpr int gate_slices(int d, int N) {
    const int n = (d + gate_slice_rows(gate_columns(N)) - 1) / gate_slice_rows(gate_columns(N));
    return n < kGateSlices ? n : kGateSlices;
}

template <int NP>
__global__ __launch_bounds__(256) void gate_part_kernel(const bf16_t* __restrict__ x, const float* __restrict__ W_gate, int T, int d, int N,
                                                        float* __restrict__ part) {
    constexpr int SUB = 64 / NP, STEP = 4 * SUB, R = STEP * kGateHeld;   // rows of a wavefront's load, of the workgroup's, of a slice
    static_assert(R == gate_slice_rows(NP), "slice");
    __shared__ float xs[kGateTokens][R];
    __shared__ float sums[kGateTokens][4][NP];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane % NP, sub = wave * SUB + lane / NP;
    const int t0 = blockIdx.y * kGateTokens, tokens = min(kGateTokens, T - t0);
    float sum[kGateTokens] = {};
    for (int r0 = blockIdx.x * R; r0 < d; r0 += gridDim.x * R) {
        float w[kGateHeld];
#pragma unroll
        for (int i = 0; i < kGateHeld; ++i) {
            const int r = r0 + i * STEP + sub;
            w[i] = r < d && col < N ? W_gate[(size_t)r * N + col] : 0.f;
        }
        __syncthreads();
        for (int p = tid; p < kGateTokens * (R / 8); p += 256) {   // d % 8 == 0
            const int t = p / (R / 8), c = p % (R / 8) * 8;
            Piece8<bf16_t> v{};
            if (t < tokens && r0 + c < d) v.load(x + (size_t)(t0 + t) * d + r0 + c);
#pragma unroll
            for (int i = 0; i < 8; ++i) xs[t][c + i] = v.at(i);
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < kGateTokens; ++t) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < kGateHeld; ++i) s = fmaf(xs[t][i * STEP + sub], w[i], s);
            sum[t] += s;
        }
    }
#pragma unroll
    for (int t = 0; t < kGateTokens; ++t) {
        float s = sum[t];
#pragma unroll
        for (int off = NP; off < 64; off <<= 1) s += __shfl_xor(s, off);
        if (lane < NP) sums[t][wave][lane] = s;
    }
    __syncthreads();
    for (int p = tid; p < tokens * NP; p += 256) {
        const int t = p / NP, c = p % NP;
        part[((size_t)(t0 + t) * gridDim.x + blockIdx.x) * NP + c] = sums[t][0][c] + sums[t][1][c] + (sums[t][2][c] + sums[t][3][c]);
    }
}

// A token by a wavefront, lane e with the logit of expert e: lane j < k has the j-th choice and its weight.
__device__ __forceinline__ void choose_experts(const ExpertsArgs& a, float logit, int lane, int& expert, float& weight) {
    float g[1] = {logit == 0.f ? 0.f : logit};   // -0 -> +0 so equal logits have equal keys
    int sel[1];
    float w[1];
    wave_topk_softmax<64, 1>(g, lane, a.N, a.k, a.inv_temperature, sel, w);
    expert = sel[0];
    weight = w[0];
}
// Token t from the partial logits
__device__ __forceinline__ void route_token(const ExpertsArgs& a, int t, int lane, int& expert, float& weight) {
    const int NP = gate_columns(a.N), slices = gate_slices(a.d, a.N), each = 64 / NP, col = lane % NP;
    const float* p = a.part + (size_t)t * slices * NP + col;
    float g[1] = {0.f};
    for (int s = lane / NP; s < slices; s += 4 * each) {
        float v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = s + u * each < slices ? p[(size_t)(s + u * each) * NP] : 0.f;
        g[0] += (v[0] + v[1]) + (v[2] + v[3]);
    }
    const float b = a.bias != nullptr && lane < a.N ? a.bias[lane] : 0.f;
    for (int off = NP; off < 64; off <<= 1) g[0] += __shfl_xor(g[0], off);
    choose_experts(a, g[0] + b, lane, expert, weight);
}
__global__ __launch_bounds__(256) void experts_route_kernel(const ExpertsArgs a) {
    const int lane = threadIdx.x & 63, t = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= a.T) return;
    int e;
    float w;
    route_token(a, t, lane, e, w);
    if (lane < a.k) {
        a.idx[t * a.k + lane] = e;
        a.w[t * a.k + lane] = w;
    }
}

// ---- which tokens an expert has: bit t of word[e], by however many of the token's slots.  LDS; all threads of the workgroup.
struct ExpertMasks { uint32_t word[kMaxAdapters][2]; };

__device__ __forceinline__ void find_masks(const ExpertsArgs& a, ExpertMasks& m) {
    int e = -1;   // T * k <= 512: up to two pairs to a thread, on their way first
    const int pairs = a.T * a.k, p0 = threadIdx.x, p1 = p0 + blockDim.x;
    if (p0 < pairs) e = a.idx[p0];
    const int e1 = p1 < pairs ? a.idx[p1] : -1;
    for (int i = threadIdx.x; i < 2 * kMaxAdapters; i += blockDim.x) m.word[i >> 1][i & 1] = 0;
    __syncthreads();
    if ((unsigned)e < (unsigned)a.N) atomicOr(&m.word[e][p0 / a.k >> 5], 1u << (p0 / a.k & 31));
    if ((unsigned)e1 < (unsigned)a.N) atomicOr(&m.word[e1][p1 / a.k >> 5], 1u << (p1 / a.k & 31));
    __syncthreads();
}
__device__ __forceinline__ uint64_t mask_of(const ExpertMasks& m, int e) { return (uint64_t)m.word[e][1] << 32 | m.word[e][0]; }
__device__ __forceinline__ int rank_in(uint64_t mask, int t) { return __popcll(mask & (((uint64_t)1 << t) - 1)); }
// an inclusive sum over the lanes (DPP: within rows of 16, then across them)
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_rows(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int wave_sums(int v) {
    v += dpp_rows<kDppRowShr + 1, 0xf>(v);
    v += dpp_rows<kDppRowShr + 2, 0xf>(v);
    v += dpp_rows<kDppRowShr + 4, 0xf>(v);
    v += dpp_rows<kDppRowShr + 8, 0xf>(v);
    v += dpp_rows<kDppBcast15, 0xa>(v);
    v += dpp_rows<kDppBcast31, 0xc>(v);
    return v;
}

// ---- weights
struct Bf16Weights {
    static constexpr int kInputs = 64, kBlockBytes = 2048, kScales = 0, kSteps = 2;   // of a K tile of 16 rows
    static constexpr int row_bytes(int d) { return d * 2; }
};
struct Mx4Weights {
    static constexpr int kInputs = 256, kBlockBytes = 2304, kScales = 1, kSteps = 8;
    static constexpr int row_bytes(int d) { return d / 2; }
};

__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p) {
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<const uint8_t*>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 |
                                            (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v));
}

// RB blocks of 16 rows of W in a wavefront's slots: the rows' bytes (see WaveOperand), then their words of scales.  Addresses are kept as they are and made
// resources for every K tile: where a ring goes from matrix to matrix the compiler keeps resources in vector registers otherwise and
// walks every load through a loop over the lanes (0.9 us to a K tile, whatever its size).
template <typename WT, int RB>
struct WeightRing {
    static constexpr int kLoads = RB * (2 + WT::kScales), kBytes = RB * WT::kBlockBytes;
    WaveOperand<RB> rows;
    __amdgpu_buffer_rsrc_t scale_rsrc;
    const uint8_t *W, *scale;
    int n, all, bytes;
    uint32_t at_scale;
    // W: the first of `n` rows of `bytes` each; scale: that matrix's, with `all` rows, of which it is row0
    __device__ __forceinline__ WeightRing(const uint8_t* W, const uint8_t* scale, int all, int row0, int n, int bytes, int lane)
        : WeightRing(bytes, lane) {
        point(W, scale, all, row0, n);
    }
    __device__ __forceinline__ WeightRing(int bytes, int lane)
        : rows(nullptr, 0, (uint32_t)bytes, lane), W(nullptr), scale(nullptr), n(0), all(0), bytes(bytes), at_scale((uint32_t)(lane & 15) * 16 + (lane >> 4) * 4) {}
    __device__ __forceinline__ void point(const uint8_t* w, const uint8_t* s, int of, int row0, int count) {
        W = w;
        n = count;
        all = of;
        if constexpr (WT::kScales) scale = s + (size_t)row0 * 16;
    }
    __device__ __forceinline__ void at_tile(int kt, int nk) {
        const int there = __builtin_amdgcn_readfirstlane(n);
        rows.mat = i8_operand(reinterpret_cast<const int8_t*>(uniform(W)), there, (uint32_t)bytes);
        rows.at_tile(kt, nk);
        if constexpr (WT::kScales)
            scale_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(uniform(scale + (size_t)(kt >> 1) * ((size_t)all * 16))), 0,
                                                           kt < nk ? (uint32_t)there * 16u : 0u, 0x00020000);
    }
    // requested as read once where rows are whole lines; where a K tile's row ends within a line, the next tile reads that line again (second product of 33
    // tokens of 28 experts, rows of 688 bytes: read once 17.2 us, kept 14.5)
    __device__ __forceinline__ void request_rows(unsigned char* slot) const {
        if (bytes % 128 == 0) {
#pragma unroll
            for (int j = 0; j < 2 * RB; ++j) rows.template request<kReadOnceI8>(slot, j);
        } else {
#pragma unroll
            for (int j = 0; j < 2 * RB; ++j) rows.template request<0>(slot, j);
        }
    }
    __device__ __forceinline__ void request(unsigned char* slot) const {
        request_rows(slot);
        if constexpr (WT::kScales)
#pragma unroll
            for (int r = 0; r < RB; ++r) mx4_scale_lds(scale_rsrc, slot + RB * 2048 + r * 256, at_scale + r * 256);
    }
};

// The fragments of a K tile's weights: 16 bytes a lane and half tile, and (4 bits) their scales
template <typename WT, int RB>
struct WeightFrags {
    u32x4 w[2][RB];
    float s[2][RB];
    __device__ __forceinline__ void read(const unsigned char* slot, int kt, int lane) {
        const int l15 = lane & 15, kq = lane >> 4;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int r = 0; r < RB; ++r)
                w[ks][r] = *reinterpret_cast<const u32x4*>(slot + r * 2048 + l15 * 128 + swz(l15, ks * 4 + kq) * 16);
        if constexpr (WT::kScales)
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                const uint32_t word = *reinterpret_cast<const uint32_t*>(slot + RB * 2048 + r * 256 + lane * 4) >> ((kt & 1) * 16);
                s[0][r] = mx4_scale(word & 255);
                s[1][r] = mx4_scale(word >> 8 & 255);
            }
    }
    // of block r in step i of kSteps
    __device__ __forceinline__ bf16x8 at(int i, int r) const {
        if constexpr (WT::kScales) return __builtin_bit_cast(bf16x8, mx4_bf16x8(w[i >> 2][r][i & 3], s[i >> 2][r]));
        else return __builtin_bit_cast(bf16x8, w[i][r]);
    }
};

// ---- tokens' rows (x or h, bf16) beside a K tile: bytes of a row there, and of R rows.  16-byte chunk c of row r lies at position
// token_chunk(r, c): a lane takes the chunk that belongs to its own 16 bytes of W, of 4 bits 4 chunks on end, one to a step.
template <typename WT> constexpr int kTokenBytes = WT::kInputs * 2;
template <typename WT>
__device__ __forceinline__ int token_chunk(int r, int c) { return WT::kScales ? c ^ (r & 15) : swz(r, c); }
template <typename WT>
__device__ __forceinline__ bf16x8 token_frag(const unsigned char* rows, int r, int kq, int i) {   // step i
    const int c = WT::kScales ? ((i >> 2) * 4 + kq) * 4 + (i & 3) : i * 4 + kq;
    return *reinterpret_cast<const bf16x8*>(rows + r * kTokenBytes<WT> + token_chunk<WT>(r, c) * 16);
}

// One load instruction of 1024 bytes of such rows: rows first, first + 1, ... by 128 or 512 bytes
template <typename WT>
struct TokenPiece {
    static constexpr int kRows = 1024 / kTokenBytes<WT>, kLanes = 64 / kRows;
    int row;             // this lane's
    uint32_t chunk;      // bytes from the K tile's first
    uint32_t voff;
    __device__ __forceinline__ void set(int first, int lane) {
        row = first + lane / kLanes;
        chunk = (uint32_t)token_chunk<WT>(row, lane % kLanes) * 16;   // an involution
    }
    // the row's first byte in the matrix, or kOutside
    __device__ __forceinline__ void point(uint32_t at) { voff = at == kOutside ? kOutside : at + chunk; }
    __device__ __forceinline__ void request(__amdgpu_buffer_rsrc_t rsrc, unsigned char* rows, int first, int kt, int nk, uint32_t ld) const {
        const uint32_t k0 = (uint32_t)kt * kTokenBytes<WT>;
        const uint32_t at = kt < nk && k0 + chunk < ld ? voff : kOutside;   // the chunks past the last input are zeros
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(rows + first * kTokenBytes<WT>), 16, at,
                                                 kt < nk ? (int)k0 : 0, 0, 0);
    }
};
__device__ __forceinline__ __amdgpu_buffer_rsrc_t token_rsrc(const bf16_t* p, int rows, int d) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(p), 0, (uint32_t)rows * (uint32_t)d * 2u, 0x00020000);
}

__device__ __forceinline__ f32x4 mfma_bf16(const bf16x8& w, const bf16x8& x, const f32x4& acc) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, acc, 0, 0, 0);
}
__device__ __forceinline__ float silu(float g) { return g / (1.f + expf(-g)); }
__device__ __forceinline__ void store_h(bf16_t* dst, const f32x4& g, const f32x4& u) {
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(silu(g[0]) * u[0], silu(g[1]) * u[1]), pack_bf16x2(silu(g[2]) * u[2], silu(g[3]) * u[3]));
}

// ---- up to 4 tokens ------------------------------------------------------------------------------------------------------------
// Columns l15 & 3 are tokens; those that are not routed to the expert have rows of zeros.
template <typename WT, int RB>
constexpr int few_slot_bytes() { return RB * WT::kBlockBytes + (kFewTokens * kTokenBytes<WT> < 1024 ? 1024 : kFewTokens * kTokenBytes<WT>); }

template <typename WT, int RB>
struct FewTile {   // a wavefront's slot: W, then the four rows
    static constexpr int kPieces = kFewTokens * kTokenBytes<WT> > 1024 ? 2 : 1, kLoads = WeightRing<WT, RB>::kLoads + kPieces;
};

// The rings of gate and up rows as one operand of two blocks
template <typename WT>
struct PairRing {
    WeightRing<WT, 1> g, u;
    __device__ __forceinline__ PairRing(int bytes, int lane) : g(bytes, lane), u(bytes, lane) {}
    __device__ __forceinline__ void at_tile(int kt, int nk) { g.at_tile(kt, nk); u.at_tile(kt, nk); }
    __device__ __forceinline__ void request(unsigned char* slot) const {   // as two blocks of one ring lie: rows, rows, scales, scales
        g.request_rows(slot);
        u.request_rows(slot + 2048);
        if constexpr (WT::kScales) {
            mx4_scale_lds(g.scale_rsrc, slot + 4096, g.at_scale);
            mx4_scale_lds(u.scale_rsrc, slot + 4352, u.at_scale);
        }
    }
};

// First product.  The tokens' rows, all of x, are in LDS for the whole workgroup; a unit is 16 channels of one expert, KS wavefronts to it, which split K,
// and the groups of a workgroup's 8 wavefronts go through the units with the loads of the next one already on their way.
constexpr int kFewWaves = 8, kFewGroups = 256, kFewDepth = 3, kFewRowsMost = 34816;   // bytes of the rows in LDS
template <typename WT>
__host__ __device__ constexpr int few_row_bytes(int d) {   // whole pieces of 1024 bytes, and K tiles; rows start 4 banks apart
    return (ceil_div(WT::row_bytes(d), 128) * kTokenBytes<WT> + 1023) / 1024 * 1024 + 16;
}
template <typename WT>
constexpr int few_up_lds(int rows_bytes, bool sums) { return kFewWaves * (kFewDepth * 2 * WT::kBlockBytes + (sums ? 2048 : 0)) + rows_bytes; }
static_assert(few_up_lds<Mx4Weights>(kFewRowsMost, true) + 1024 <= 160 * 1024, "LDS");

// The gate of one token by every workgroup for itself, from x in LDS (zeros at `pad`): two rows of W_gate to a thread and step, all steps on their way at
// once, up to two passes of them.  A layer of 28 experts of 1024 inputs takes 14.8 us so, with gate_part_kernel in front 16.6, of 8 of 1024 14.0 and
// 17.5; two passes, 64 experts of 1024, 19.4 and 19.9.  Of more tokens every workgroup has too much to add up (4 of 8 experts of 4096: 24.8 and 20.6).
constexpr int kGateHere = 65536, kGatePairs = 32, kGatePass = 2 * kGatePairs * kFewWaves * 64;
__device__ __forceinline__ void load_gate(const ExpertsArgs& a, int lane, int wave, int pass, float (&w)[2 * kGatePairs]) {
    const int NP = gate_columns(a.N), col = lane & (NP - 1), each = 64 / NP;
    const auto W = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(a.W_gate), 0, (uint32_t)(a.d * a.N) * 4u, 0x00020000);   // zeros behind the last row
    const uint32_t row = (uint32_t)a.N * 4, step = 2 * kFewWaves * each * row;
    uint32_t at = col < a.N ? 2 * ((pass * kGatePairs * kFewWaves + wave) * each + lane / NP) * row + col * 4 : kOutside;
#pragma unroll
    for (int i = 0; i < kGatePairs; ++i, at += step) {
        w[2 * i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(W, at, 0, 0));
        w[2 * i + 1] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(W, at + row, 0, 0));
    }
}
__device__ __forceinline__ float gate_here(const ExpertsArgs& a, const float (&w)[2 * kGatePairs], const unsigned char* x, int pad, int lane, int wave, int pass) {
    const int NP = gate_columns(a.N), each = 64 / NP;
    int at = ((pass * kGatePairs * kFewWaves + wave) * each + lane / NP) * 4;
    float s[4] = {};
#pragma unroll
    for (int i = 0; i < kGatePairs; ++i, at += kFewWaves * each * 4) {
        const uint32_t v = *reinterpret_cast<const uint32_t*>(x + min(at, pad));
        s[i & 3] = fmaf(__uint_as_float(v << 16), w[2 * i], s[i & 3]);
        s[i & 3] = fmaf(__uint_as_float(v & 0xffff0000u), w[2 * i + 1], s[i & 3]);
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
}

template <typename WT, int KS>
__global__ __launch_bounds__(kFewWaves * 64) void experts_few_up_kernel(const ExpertsArgs a) {
    constexpr int D = kFewDepth, NL = 2 * (2 + WT::kScales), kSlot = 2 * WT::kBlockBytes, GROUPS = kFewWaves / KS;
    static_assert((D - 1) * NL < 64, "vmcnt");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ ExpertMasks masks;
    __shared__ uint32_t list[kMaxAdapters];   // the experts in use: id | tokens << 8 | first row of h << 16
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, kq = lane >> 4;
    unsigned char* const ring = smem + wave * D * kSlot;
    f32x4* const sums = reinterpret_cast<f32x4*>(smem + kFewWaves * D * kSlot);
    unsigned char* const rows = smem + kFewWaves * (D * kSlot + (KS > 1 ? 2048 : 0));
    const int row_bytes = few_row_bytes<WT>(a.d);
    {   // x, before anything is known of the routing
        const auto x = token_rsrc(a.x, a.T, a.d);
        const int per = row_bytes / 1024;
        for (int p = wave; p < a.T * per; p += kFewWaves) {
            const int t = p / per, c = (p - t * per) * 1024 + lane * 16;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                x, (__attribute__((address_space(3))) void*)(rows + t * row_bytes + (p - t * per) * 1024), 16,
                c < a.d * 2 ? (uint32_t)t * (uint32_t)a.d * 2u + (uint32_t)c : kOutside, 0, 0, 0);   // zeros behind a row
        }
    }
    if (a.part != nullptr) {   // every workgroup routes; the first one says how
        int e = -1;
        float w = 0.f;
        if (a.W_gate != nullptr) {
            float* const logits = reinterpret_cast<float*>(smem);   // in the rings' place
            const int NP = gate_columns(a.N);
            float held[2 * kGatePairs];
            load_gate(a, lane, wave, 0, held);
            const float b = a.bias != nullptr && lane < a.N ? a.bias[lane] : 0.f;
            if (tid < 4) reinterpret_cast<uint32_t*>(rows + row_bytes - 16)[tid] = 0;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // x
            __syncthreads();
            float sum = gate_here(a, held, rows, row_bytes - 16, lane, wave, 0);
            if (a.d * NP > kGatePass) {
                load_gate(a, lane, wave, 1, held);
                sum += gate_here(a, held, rows, row_bytes - 16, lane, wave, 1);
            }
            for (int off = NP; off < 64; off <<= 1) sum += __shfl_xor(sum, off);
            if (lane < NP) logits[wave * NP + lane] = sum;
            __syncthreads();
            if (wave == 0) {
                float g = 0.f;
                if (lane < NP)
#pragma unroll
                    for (int v = 0; v < kFewWaves; ++v) g += logits[v * NP + lane];
                choose_experts(a, g + b, lane, e, w);
            }
        } else if (wave < a.T) {
            route_token(a, wave, lane, e, w);
        }
        if (tid < 2 * kMaxAdapters) masks.word[tid >> 1][tid & 1] = 0;
        __syncthreads();
        if (wave < a.T && lane < a.k) {
            if ((unsigned)e < (unsigned)a.N) atomicOr(&masks.word[e][0], 1u << wave);
            if (blockIdx.x == 0) {
                a.idx[wave * a.k + lane] = e;
                a.w[wave * a.k + lane] = w;
            }
        }
        __syncthreads();
    } else {
        find_masks(a, masks);
    }
    const uint64_t mine = lane < a.N ? mask_of(masks, lane) : 0;
    const uint64_t active = __ballot(mine != 0);
    if (wave == 0) {
        const int n = __popcll(mine), at = wave_sums(n) - n;
        if (n != 0) list[rank_in(active, lane)] = (uint32_t)lane | (uint32_t)mine << 8 | (uint32_t)at << 16;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wavefront's part of x
    __syncthreads();

    const int group = wave / KS, kp = wave % KS, each = ceil_div(a.f, 16), total = __popcll(active) * each;
    const int slot0 = xcd_order(blockIdx.x, kFewGroups), stride = kFewGroups * GROUPS;   // a unit to every workgroup, then a second one
    const int mine_at = group * kFewGroups;
    const int bytes = WT::row_bytes(a.d), nk = ceil_div(bytes, 128);
    struct Unit { int e, first, c0, n; uint32_t tokens; };
    auto unit_at = [&](int u) {
        const int i = u / each, c0 = (u - i * each) * 16;
        const uint32_t v = (uint32_t)__builtin_amdgcn_readfirstlane((int)list[i]);
        return Unit{(int)(v & 255), (int)(v >> 16), c0, min(16, a.f - c0), v >> 8 & 255};
    };
    PairRing<WT> w(bytes, lane);
    int req_u = slot0 + mine_at, req_kt = kp, req_end = 0, req_at = 0;   // req_end: 0 where there are no more
    auto point = [&] {
        const Unit m = unit_at(req_u);
        const uint8_t* W = a.W1 + ((size_t)m.e * 2 * a.f + m.c0) * bytes;
        const uint8_t* S = WT::kScales ? a.s1 + (size_t)m.e * mx4_scale_bytes(2 * a.f, a.d) : nullptr;
        w.g.point(W, S, 2 * a.f, m.c0, m.n);
        w.u.point(W + (size_t)a.f * bytes, S, 2 * a.f, a.f + m.c0, m.n);
        req_end = nk;
    };
    if (req_u < total && kp < nk) point();
    auto request = [&] {
        w.at_tile(req_kt, req_end);
        w.request(ring + req_at * kSlot);
        req_at = req_at + 1 == D ? 0 : req_at + 1;
        req_kt += KS;
        if (req_kt >= req_end && req_end > 0) {
            req_kt = kp;
            req_u += stride;
            if (req_u < total) point();
            else req_end = 0;
        }
    };
#pragma unroll
    for (int i = 0; i < D; ++i) request();
    const unsigned char* const mine_row = rows + (l15 % a.T) * row_bytes;   // columns past the last token: another's, not kept
    int at = 0;
    for (int u0 = slot0; u0 < total; u0 += stride) {   // the same rounds for all groups
        const int u = u0 + mine_at;
        f32x4 ag = {0.f, 0.f, 0.f, 0.f}, au = {0.f, 0.f, 0.f, 0.f};
        const int end = u < total ? nk : 0;
        for (int kt = kp; kt < end; kt += KS) {
            unsigned char* const slot = ring + at * kSlot;
            at = at + 1 == D ? 0 : at + 1;
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * NL) : "memory");
            WeightFrags<WT, 2> wf;
            wf.read(slot, kt, lane);
            bf16x8 xf[WT::kSteps];
#pragma unroll
            for (int i = 0; i < WT::kSteps; ++i) {
                const int c = WT::kScales ? ((i >> 2) * 4 + kq) * 4 + (i & 3) : i * 4 + kq;
                xf[i] = *reinterpret_cast<const bf16x8*>(mine_row + kt * kTokenBytes<WT> + c * 16);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slot is read
            request();
#pragma unroll
            for (int i = 0; i < WT::kSteps; ++i) {
                ag = mfma_bf16(wf.at(i, 0), xf[i], ag);
                au = mfma_bf16(wf.at(i, 1), xf[i], au);
            }
        }
        if constexpr (KS > 1) {
            sums[wave * 128 + lane] = ag;
            sums[wave * 128 + 64 + lane] = au;
            __syncthreads();
            if (kp == 0) {
#pragma unroll
                for (int v = 1; v < KS; ++v) {
                    ag += sums[(wave + v) * 128 + lane];
                    au += sums[(wave + v) * 128 + 64 + lane];
                }
            }
        }
        if (kp == 0 && u < total) {
            const Unit m = unit_at(u);
            if (l15 < a.T && (m.tokens >> l15 & 1) && kq * 4 < m.n)   // f % 8 == 0
                store_h(a.h + (size_t)(m.first + rank_in(m.tokens, l15)) * a.f + m.c0 + kq * 4, ag, au);
        }
        if constexpr (KS > 1) __syncthreads();   // the sums are read
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may land after the end
}

// Second product.  The wavefronts split K (KS of them), and where there are few channels so do `splits` workgroups, whose sums then leave as y[part][T][d];
// sequence numbers run over the experts in use and their K tiles.
template <typename WT, int KS, int D>
__global__ __launch_bounds__(KS * 64) void experts_few_down_kernel(const ExpertsArgs a, int splits) {
    constexpr int NL = FewTile<WT, 1>::kLoads, NP = FewTile<WT, 1>::kPieces, kSlot = few_slot_bytes<WT, 1>();
    static_assert((D - 1) * NL < 64, "vmcnt");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ ExpertMasks masks;
    __shared__ int list[kMaxAdapters][2];                  // the experts in use and their first rows of h
    __shared__ float weight[kMaxAdapters][kFewTokens];
    __shared__ int ids[kFewTokens * kMaxTopK];
    __shared__ float ws[kFewTokens * kMaxTopK];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, kq = lane >> 4;
    if (tid < a.T * a.k) {
        ids[tid] = a.idx[tid];
        ws[tid] = a.w[tid];
    }
    find_masks(a, masks);
    const uint64_t mine = lane < a.N ? mask_of(masks, lane) : 0;
    const uint64_t active = __ballot(mine != 0);
    const int count = __popcll(active);
    if (wave == 0) {
        const int sums = wave_sums(__popcll(mine));
        if (mine != 0) {
            const int i = rank_in(active, lane);
            list[i][0] = lane;
            list[i][1] = sums - __popcll(mine);
            for (int t = 0; t < kFewTokens; ++t) {
                float w = 0.f;
                for (int j = 0; j < a.k && t < a.T; ++j)
                    if (ids[t * a.k + j] == lane) w += ws[t * a.k + j];
                weight[i][t] = w;
            }
        }
    }
    __syncthreads();
    const int id = xcd_order(blockIdx.x, gridDim.x), part = id % splits, c0 = id / splits * 16, n = min(16, a.d - c0);
    unsigned char* const ring = smem + wave * D * kSlot;
    const int bytes = WT::row_bytes(a.f), nk = ceil_div(bytes, 128), share = ceil_div(nk, splits);
    const int kt0 = part * share + wave, kt1 = min(nk, part * share + share);   // this wavefront's: every KS-th of an expert's
    const int per = kt0 < kt1 ? (kt1 - 1 - kt0) / KS + 1 : 0, steps = per * count;
    const auto h = token_rsrc(a.h, a.T * a.k, a.f);
    WeightRing<WT, 1> w(a.W2, a.s2, a.d, c0, n, bytes, lane);
    TokenPiece<WT> piece[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) piece[i].set(i * TokenPiece<WT>::kRows, lane);
    int req_i = 0, req_kt = kt0;   // next request: expert of the list, K tile
    auto point = [&](int i) {
        const int e = __builtin_amdgcn_readfirstlane(list[i][0]), row = __builtin_amdgcn_readfirstlane(list[i][1]);
        const uint32_t tokens = masks.word[e][0];
        w.point(a.W2 + ((size_t)e * a.d + c0) * bytes, WT::kScales ? a.s2 + (size_t)e * mx4_scale_bytes(a.d, a.f) : nullptr, a.d, c0, n);
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int t = piece[p].row;
            piece[p].point(t < kFewTokens && (tokens >> t & 1) ? (uint32_t)(row + rank_in(tokens, t)) * (uint32_t)a.f * 2u : kOutside);
        }
    };
    if (count > 0) point(0);
    auto request = [&](unsigned char* slot) {
        const int end = req_i < count && per > 0 ? kt1 : 0;
        w.at_tile(req_kt, end);
        w.request(slot);
#pragma unroll
        for (int p = 0; p < NP; ++p)
            piece[p].request(h, slot + WT::kBlockBytes, p * TokenPiece<WT>::kRows, req_kt, end, (uint32_t)a.f * 2u);
        req_kt += KS;
        if (req_kt >= kt1 && req_i < count) {
            req_kt = kt0;
            if (++req_i < count) point(req_i);
        }
    };
#pragma unroll
    for (int i = 0; i < D; ++i) request(ring + i * kSlot);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f}, total = {0.f, 0.f, 0.f, 0.f};
    int at = 0, i = 0, kt = kt0;
    for (int s = 0; s < steps; ++s) {
        unsigned char* const slot = ring + at * kSlot;
        at = at + 1 == D ? 0 : at + 1;
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * NL) : "memory");
        WeightFrags<WT, 1> wf;
        wf.read(slot, kt, lane);
        bf16x8 xf[WT::kSteps];
#pragma unroll
        for (int j = 0; j < WT::kSteps; ++j) xf[j] = token_frag<WT>(slot + WT::kBlockBytes, l15 & (kFewTokens - 1), kq, j);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slot is read
        request(slot);
#pragma unroll
        for (int j = 0; j < WT::kSteps; ++j) acc = mfma_bf16(wf.at(j, 0), xf[j], acc);
        kt += KS;
        if (kt >= kt1) {   // the expert's last: its sum with the token's weight
            const int t = l15 & (kFewTokens - 1);
            const float wt = weight[i][t];
            const bool routed = masks.word[list[i][0]][0] >> t & 1;   // a column of zeros may meet a NaN in the weights
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                total[c] += routed ? wt * acc[c] : 0.f;
                acc[c] = 0.f;
            }
            kt = kt0;
            ++i;
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may land in what follows
    __syncthreads();
    f32x4* const sums = reinterpret_cast<f32x4*>(smem);
    sums[wave * 64 + lane] = total;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int v = 1; v < KS; ++v) total += sums[v * 64 + lane];
    if (l15 >= a.T || l15 >= kFewTokens || kq * 4 >= n) return;
    const size_t o = (size_t)l15 * a.d + c0 + kq * 4;
    if (splits > 1) {
        *reinterpret_cast<f32x4*>(a.y + (size_t)part * a.T * a.d + o) = total;
        return;
    }
    float v[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = a.scale * total[c] + (a.base != nullptr ? (float)a.base[o + c] : 0.f);
    *reinterpret_cast<uint2*>(a.out + o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

__global__ __launch_bounds__(256) void experts_few_sum_kernel(const ExpertsArgs a, int splits) {   // 4 channels of a token to a thread
    const size_t o = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4, all = (size_t)a.T * a.d;
    if (o >= all) return;
    f32x4 sum = *reinterpret_cast<const f32x4*>(a.y + o);
    for (int p = 1; p < splits; ++p) sum += *reinterpret_cast<const f32x4*>(a.y + (size_t)p * all + o);
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a.scale * sum[i] + (a.base != nullptr ? (float)a.base[o + i] : 0.f);
    *reinterpret_cast<uint2*>(a.out + o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

// ---- more tokens -----------------------------------------------------------------------------------------------------------------
// Blocks of R = 16 TB tokens of an expert; w wavefronts of a workgroup's 8 take 16 rows of gate and up (32 rows of W2) each, and all share the
// tokens' rows.  A workgroup has every grid-th (tile, block), and its loads run on from one into the next.
constexpr int kManyWaves = 8, kManyThreads = kManyWaves * 64, kManyGroups = 256, kManySplits = 4;
static_assert(kManyThreads >= kExpertsMaxTokens * kMaxTopK, "a pair to a thread");

// What a launch of 256 workgroups does: w, and (down) the parts that K is cut into.  The choice is the one that takes the least by
//   rounds * K tiles of a part * time of one + parts
// us.  A K tile of w wavefronts took, 4 bits and blocks of 16 tokens (20 tokens of 16 experts, 4096 and 2048 wide), 0.54, 0.57, 0.62, 0.69, 0.85, 0.91,
// 0.94, 1.24 us for w = 1 to 8, and with blocks of 32 (64 tokens of 8 experts, 4096 and 14336) 0.70, 0.74, 0.83, 0.97, 1.25, 1.32, 1.45, 1.6.
// Calls of 33 tokens of 28 experts, 2080 and 1376 wide, with w = 4, 5 and 8 for the first product 51.6, 49.4, 55.5; of 64 of 8, 4096 and 14336, w = 4, 7, 8
// 166, 150, 159, and the second product with w = 8 whole and in two and four parts 180, 152, 154.  The model is that of 4 bits
// for both kinds of weights: of 16 calls of 6 to 64 tokens of 4 to 64 experts the best of all w and parts takes 0 to 2 % less than the choice in 4 bits and 0 to 8 % in
// bf16, where fewer wavefronts would do (first product of 13 tokens of 8 experts, 4096 and 3584, 129 us, with w = 2 119; 32 tokens 127 and 120).
struct Tiling { int waves, splits; };
__device__ __forceinline__ Tiling choose_tiling(int blocks, int units, int nk, bool may_split, int lane) {   // a wavefront; units: of channels
    const int w = (lane & 7) + 1, splits = 1 << (lane >> 3 & 3);
    const int items = blocks * ((units + w - 1) / w) * splits;
    const float tile = w <= 4 ? 0.49f + 0.05f * (float)w : 0.5f + 0.07f * (float)w;
    const float us = (float)((items + kManyGroups - 1) / kManyGroups) * (float)((nk + splits - 1) / splits) * tile + (float)splits;
    const bool there = lane < 8 || (may_split && lane < 24 && splits <= kManySplits && nk >= 4 * splits);   // no part is empty
    // the least, of equal ones the first lane's; positive floats compare as whole numbers
    uint32_t best = there ? (__float_as_uint(us) & ~31u) | (uint32_t)(lane & 31) : 0x7f800000u;
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) best = min(best, (uint32_t)__shfl_xor((int)best, off));
    const int at = __builtin_amdgcn_readfirstlane((int)(best & 31));
    return {(at & 7) + 1, 1 << (at >> 3 & 3)};
}

// The plan of a call, in the workspace for the launches behind the first
struct Plan {
    int blocks, splits;   // splits: of the second product
    int up_waves, down_waves;
    uint32_t block[kMaxAdapters + kExpertsMaxTokens * kMaxTopK / 16];   // expert | tokens << 8 | first row of h and y << 16
    int16_t row[kExpertsMaxTokens * kMaxTopK];                           // of pair (t, j), -1: none
};
size_t experts_plan_bytes() { return sizeof(Plan); }

static_assert(kRouteTokens * kMaxTopK <= 2 * kMaxAdapters, "room");

// All threads of a workgroup.  token: of a row of h.  first: room for the first row of every expert.  to: where the plan goes, or nullptr.
template <typename WT, int R>
__device__ __forceinline__ void make_plan(const ExpertsArgs& a, Plan& plan, ExpertMasks& masks, int (&first)[2 * kMaxAdapters],
                                          uint8_t (&token)[kExpertsMaxTokens * kMaxTopK], Plan* to) {
    const int lane = threadIdx.x & 63, pairs = a.T * a.k, p = threadIdx.x;   // a pair each
    const int t = p / a.k;
    int e = -1;
    if (a.part != nullptr && a.T <= kRouteTokens) {   // two tokens to a wavefront; the first workgroup says how
        int* const ids = first;   // of kRouteTokens * kMaxTopK pairs, and room for as many
        for (int i = threadIdx.x >> 6; i < a.T; i += kManyWaves) {
            int choice;
            float w;
            route_token(a, i, lane, choice, w);
            if (lane < a.k) {
                ids[i * a.k + lane] = choice;
                if (to != nullptr) {
                    a.idx[i * a.k + lane] = choice;
                    a.w[i * a.k + lane] = w;
                }
            }
        }
        __syncthreads();
        if (p < pairs) e = ids[p];
    } else if (p < pairs) {
        e = a.idx[p];
    }
    const bool there = (unsigned)e < (unsigned)a.N;
    for (int i = threadIdx.x; i < 2 * kMaxAdapters; i += kManyThreads) masks.word[i >> 1][i & 1] = 0;
    __syncthreads();
    if (there) atomicOr(&masks.word[e][t >> 5], 1u << (t & 31));
    __syncthreads();
    if (threadIdx.x < 64) {
        const int n = lane < a.N ? __popcll(mask_of(masks, lane)) : 0, mine = (n + R - 1) / R;
        const int at = wave_sums(n) - n, end = wave_sums(mine);
        first[lane] = at;
        for (int i = 0; i < mine; ++i) plan.block[end - mine + i] = (uint32_t)lane | (uint32_t)min(R, n - i * R) << 8 | (uint32_t)(at + i * R) << 16;
        const int blocks = __builtin_amdgcn_readlane(end, 63);
        const Tiling up = choose_tiling(blocks, ceil_div(a.f, 16), ceil_div(WT::row_bytes(a.d), 128), false, lane);
        const Tiling down = choose_tiling(blocks, ceil_div(a.d, 32), ceil_div(WT::row_bytes(a.f), 128), true, lane);
        if (lane == 0) {
            plan.blocks = blocks;
            plan.up_waves = up.waves;
            plan.down_waves = down.waves;
            plan.splits = down.splits;
        }
    }
    __syncthreads();
    const int row = there ? first[e] + rank_in(mask_of(masks, e), t) : -1;
    if (there) token[row] = (uint8_t)t;
    if (p < pairs) plan.row[p] = (int16_t)row;
    __syncthreads();
    if (to != nullptr)
        for (int i = threadIdx.x; i < (int)(sizeof(Plan) / 4); i += kManyThreads) reinterpret_cast<uint32_t*>(to)[i] = reinterpret_cast<const uint32_t*>(&plan)[i];
}
struct Block { int e, count, first; };
__device__ __forceinline__ Block unpack_block(uint32_t v) {
    const uint32_t u = (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
    return {(int)(u & 255), (int)(u >> 8 & 255), (int)(u >> 16)};
}

// A slot with room for the rows of MOST wavefronts, and as many of them as LDS has room for
template <typename WT, int TB, int MOST>
constexpr int many_slot_bytes() { return MOST * 2 * WT::kBlockBytes + TB * 16 * kTokenBytes<WT>; }
constexpr int kManyRings = 160 * 1024 - 2048;   // what the plan leaves
template <typename WT, int TB, int MOST>
constexpr int many_depth() { return kManyRings / many_slot_bytes<WT, TB, MOST>() < 8 ? kManyRings / many_slot_bytes<WT, TB, MOST>() : 8; }
template <typename WT, int TB>
constexpr int many_lds() {
    constexpr int a = many_depth<WT, TB, 4>() * many_slot_bytes<WT, TB, 4>(), b = many_depth<WT, TB, 8>() * many_slot_bytes<WT, TB, 8>();
    return a > b ? a : b;
}

// The second 16 tokens are multiplied whether there are any or not: with a branch around their MFMAs the compiler moves accumulators right behind
// the branch and leaves out the wait states for it (ROCm 7.2; tests/test_experts_host.py looks for that).  For the same reason wavefronts
// without channels, which only load tokens, have a loop of their own.
// UP: channels of h from the rows of x, the first launch; otherwise channels of y from those of h.  MOST: of the wavefronts that have channels,
// 4 or 8: up to 4, which have the shorter K tiles, run on deeper rings.
template <typename WT, bool UP, int TB, int MOST>
__device__ __forceinline__ void many_tiles(const ExpertsArgs& a, const Plan& plan, const uint8_t (&token)[kExpertsMaxTokens * kMaxTopK],
                                           unsigned char* smem, int waves) {
    constexpr int WV = kManyWaves, R = TB * 16, RB = 2, kSlot = many_slot_bytes<WT, TB, MOST>(), D = many_depth<WT, TB, MOST>();
    constexpr int kTokens = MOST * RB * WT::kBlockBytes, kRowsPer = TokenPiece<WT>::kRows;   // where the tokens' rows lie in a slot
    constexpr int PIECES = R / kRowsPer, NP = PIECES < WV ? 1 : PIECES / WV, NL = RB * (2 + WT::kScales) + NP;
    constexpr int CW = UP ? 16 : 32;   // channels of a wavefront
    static_assert(D >= 3 && (D - 2) * NL < 64, "vmcnt");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, kq = lane >> 4;
    const int K = UP ? a.d : a.f, C = UP ? a.f : a.d;   // inputs, channels
    const int splits = UP ? 1 : __builtin_amdgcn_readfirstlane(plan.splits);
    const int bytes = WT::row_bytes(K), nk = ceil_div(bytes, 128), per = ceil_div(nk, splits);
    const int nb = __builtin_amdgcn_readfirstlane(plan.blocks) * splits, total = nb * ceil_div(C, waves * CW);   // 0: no token has an expert
    // workgroups: as many on every XCD, each with the same number of items but for some that have one less
    const int G = ceil_div(total, max(ceil_div(total, kManyGroups), 1));
    if (total == 0 || (int)blockIdx.x >= G) return;
    const int start = xcd_order(blockIdx.x, G);

    struct Item { int col, part; Block b; };
    auto item_at = [&](int i) {   // tiles of one column for all blocks, of a block for all parts
        const int col = i / nb, rest = i - col * nb, b = rest / splits;
        return Item{col, rest - b * splits, unpack_block(plan.block[b])};
    };
    std::conditional_t<UP, PairRing<WT>, WeightRing<WT, RB>> ring(bytes, lane);
    const auto rows = UP ? token_rsrc(a.x, a.T, a.d) : token_rsrc(a.h, a.T * a.k, a.f);
    auto first_row = [&](int i) { return ((i * WV + wave) % PIECES) * kRowsPer; };   // fewer pieces than wavefronts: some twice
    TokenPiece<WT> piece[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) piece[i].set(first_row(i), lane);

    int req_item = start, req_kt, req_end, req_at = 0;   // next request: K tile of an item; behind the last one req_kt = req_end = 0
    auto point = [&] {
        const Item m = item_at(req_item);
        const int c0 = (m.col * waves + wave) * CW, n = max(min(CW, C - c0), 0);
        req_kt = m.part * per;
        req_end = min(nk, req_kt + per);
        if constexpr (UP) {
            const uint8_t* W = a.W1 + ((size_t)m.b.e * 2 * a.f + c0) * bytes;
            const uint8_t* S = WT::kScales ? a.s1 + (size_t)m.b.e * mx4_scale_bytes(2 * a.f, a.d) : nullptr;
            ring.g.point(W, S, 2 * a.f, c0, n);
            ring.u.point(W + (size_t)a.f * bytes, S, 2 * a.f, a.f + c0, n);
        } else {
            ring.point(a.W2 + ((size_t)m.b.e * a.d + c0) * bytes, WT::kScales ? a.s2 + (size_t)m.b.e * mx4_scale_bytes(a.d, a.f) : nullptr, a.d, c0, n);
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int r = piece[i].row;
            const uint32_t row = UP ? token[m.b.first + min(r, m.b.count - 1)] : (uint32_t)(m.b.first + r);
            piece[i].point(r < m.b.count ? row * (uint32_t)K * 2u : kOutside);
        }
    };
    point();
    auto request = [&](auto with_weights) {
        unsigned char* const slot = smem + req_at * kSlot;
        req_at = req_at + 1 == D ? 0 : req_at + 1;
        if constexpr (decltype(with_weights)::value) {
            ring.at_tile(req_kt, req_end);
            ring.request(slot + wave * RB * WT::kBlockBytes);
        }
#pragma unroll
        for (int i = 0; i < NP; ++i)
            piece[i].request(rows, slot + kTokens, first_row(i), req_kt, req_end, (uint32_t)K * 2u);
        if (++req_kt >= req_end && req_end > 0) {
            req_item += G;
            if (req_item < total) point();
            else req_kt = req_end = 0;
        }
    };
    if (wave >= waves) {
#pragma unroll
        for (int i = 0; i < D - 1; ++i) request(std::false_type{});
        for (int item = start; item < total; item += G) {
            const int part = item % splits;   // nb is a multiple of splits
            for (int kt = part * per; kt < min(nk, part * per + per); ++kt) {
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((D - 2) * NP) : "memory");
                request(std::false_type{});
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may land after the end
        return;
    }
#pragma unroll
    for (int i = 0; i < D - 1; ++i) request(std::true_type{});
    f32x4 acc[TB][RB];
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int r = 0; r < RB; ++r) acc[t][r] = f32x4{0.f, 0.f, 0.f, 0.f};
    int at = 0;
    for (int item = start; item < total; item += G) {
        const Item m = item_at(item);
        const int end = min(nk, m.part * per + per);
        for (int kt = m.part * per; kt < end; ++kt) {
            // this wavefront's part of the tile has landed, and so, behind the barrier, the others'; the slot before is read by all
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((D - 2) * NL) : "memory");
            const unsigned char* const slot = smem + at * kSlot;
            at = at + 1 == D ? 0 : at + 1;
            WeightFrags<WT, RB> w;
            w.read(slot + wave * RB * WT::kBlockBytes, kt, lane);
            const unsigned char* const tokens = slot + kTokens;
            bf16x8 xf[TB][WT::kSteps];
#pragma unroll
            for (int i = 0; i < WT::kSteps; ++i)
#pragma unroll
                for (int t = 0; t < TB; ++t) xf[t][i] = token_frag<WT>(tokens, t * 16 + l15, kq, i);
            __builtin_amdgcn_sched_barrier(0);
            request(std::true_type{});   // while the fragments are on their way
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < WT::kSteps; ++i) {
                bf16x8 wf[RB];
#pragma unroll
                for (int r = 0; r < RB; ++r) wf[r] = w.at(i, r);
#pragma unroll
                for (int t = 0; t < TB; ++t)
#pragma unroll
                    for (int r = 0; r < RB; ++r) acc[t][r] = mfma_bf16(wf[r], xf[t][i], acc[t][r]);
            }
        }
        const int c0 = (m.col * waves + wave) * CW, n = min(CW, C - c0);
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            const int r = t * 16 + l15;
            if constexpr (UP) {
                if (r < m.b.count && kq * 4 < n) store_h(a.h + (size_t)(m.b.first + r) * a.f + c0 + kq * 4, acc[t][0], acc[t][1]);
            } else {
                float* const y = a.y + (size_t)m.part * ((size_t)a.T * a.k * a.d) + (size_t)(m.b.first + r) * a.d + c0 + kq * 4;
#pragma unroll
                for (int q = 0; q < RB; ++q)
                    if (r < m.b.count && q * 16 + kq * 4 < n) *reinterpret_cast<f32x4*>(y + q * 16) = acc[t][q];
            }
#pragma unroll
            for (int q = 0; q < RB; ++q) acc[t][q] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may land after the end
}

template <typename WT, bool UP, int TB>
__global__ __launch_bounds__(kManyThreads) void experts_many_kernel(const ExpertsArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ Plan plan;
    __shared__ uint8_t token[kExpertsMaxTokens * kMaxTopK];
    const int tid = threadIdx.x;
    if constexpr (UP) {
        // masks and the experts' first rows are in the rings' place
        make_plan<WT, TB * 16>(a, plan, *reinterpret_cast<ExpertMasks*>(smem), *reinterpret_cast<int(*)[2 * kMaxAdapters]>(smem + sizeof(ExpertMasks)), token,
                               blockIdx.x == 0 ? reinterpret_cast<Plan*>(a.plan) : nullptr);
        __syncthreads();
    } else {
        for (int i = tid; i < (int)(offsetof(Plan, row) / 4); i += kManyThreads)
            reinterpret_cast<uint32_t*>(&plan)[i] = reinterpret_cast<const uint32_t*>(a.plan)[i];
        __syncthreads();
    }
    const int waves = __builtin_amdgcn_readfirstlane(UP ? plan.up_waves : plan.down_waves);
    if (waves <= 4) many_tiles<WT, UP, TB, 4>(a, plan, token, smem, waves);
    else many_tiles<WT, UP, TB, 8>(a, plan, token, smem, waves);
}

// out[t] = base[t] + scale * sum_j w[t,j] * y[row of (t, j)], the parts of y added first; a token and 1024 channels to a workgroup
__global__ __launch_bounds__(256) void experts_sum_kernel(const ExpertsArgs a) {
    const Plan* const plan = reinterpret_cast<const Plan*>(a.plan);
    const int t = blockIdx.y, c = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (c >= a.d) return;
    const int splits = plan->splits;
    const size_t part = (size_t)a.T * a.k * a.d;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < a.k; ++j) {
        const int row = plan->row[t * a.k + j];
        if (row < 0) continue;
        const float w = a.w[t * a.k + j];
        const float* const y = a.y + (size_t)row * a.d + c;
        f32x4 v = *reinterpret_cast<const f32x4*>(y);
        for (int s = 1; s < splits; ++s) v += *reinterpret_cast<const f32x4*>(y + (size_t)s * part);
        sum += w * v;
    }
    const size_t o = (size_t)t * a.d + c;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a.scale * sum[i] + (a.base != nullptr ? (float)a.base[o + i] : 0.f);
    *reinterpret_cast<uint2*>(a.out + o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

template <typename K>
static hipError_t start(K kern, int grid, int threads, int lds, const ExpertsArgs& a, hipStream_t stream) {
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(kern), lds);
    if (e != hipSuccess) return e;
    kern<<<grid, threads, lds, stream>>>(a);
    return hipGetLastError();
}
template <typename WT, int KS, int D>
constexpr int few_down_lds() { return KS * D * few_slot_bytes<WT, 1>(); }
constexpr int kFewDownWaves = 8;
// K tiles of a ring.  Where there are more workgroups than CUs shorter rings let two share one: a token of 2 experts of 4608 and 5888 in 4 bits 31.0 us, in
// two rounds of the longer rings 34.9, of 5120 and 4096 in bf16 55.2 and 61.9.
template <typename WT> constexpr int kFewDownDepth = WT::kScales ? 4 : 5;    // one workgroup to a CU
template <typename WT> constexpr int kFewDownDepth2 = WT::kScales ? 2 : 3;   // two
static_assert(2 * (few_down_lds<Mx4Weights, kFewDownWaves, 2>() + 4096) <= 160 * 1024 && 2 * (few_down_lds<Bf16Weights, kFewDownWaves, 3>() + 4096) <= 160 * 1024, "LDS");

// Wavefronts to a unit of the first product: rounds * K tiles of each, and a round's sum in LDS as half a K tile.  1, 2, 4 and 8 took 19.3, 15.1, 13.3
// and 13.4 us for a token of 2 experts of 4096 and 1024 in 4 bits (it takes 4), 42.1, 42.9, 43.0 and 45.5 for 14336 channels (1).
static int few_up_split(int units, int nk) {
    int best = 1;
    float least = 0.f;
    for (int KS = 1; KS <= kFewWaves; KS *= 2) {
        const float us = (float)ceil_div(units, kFewGroups * kFewWaves / KS) * ((float)ceil_div(nk, KS) + (KS > 1 ? 0.5f : 0.f));
        if (KS == 1 || us < least) { least = us; best = KS; }
    }
    return best;
}
// Workgroups to a tile of the second product: rounds * K tiles of a wavefront, 0.4 us each (of 4 bits 0.75), and a launch of 3.5 us that adds the parts.
// 1, 2 and 4 took 40.3, 31.9 and 28.4 us for 8 experts of 512 and 4096 in bf16 (it takes 4), 24.8, 21.8 and 20.7 in 4 bits (2: 4 would leave
// wavefronts without a K tile), 39.2, 44.3 and 53.7 for 8 of 4096 and 1024 in bf16 (1).
template <typename WT>
static int few_down_split(int tiles, int experts, int nk) {
    constexpr float kTile = WT::kScales ? 0.75f : 0.4f;
    int best = 1;
    float least = 0.f;
    for (int S = 1; S <= kManySplits; S *= 2) {
        const float us = (float)ceil_div(tiles * S, 256) * (float)(experts * ceil_div(ceil_div(nk, S), kFewDownWaves)) * kTile + (S > 1 ? 3.5f : 0.f);
        if (S > 1 && nk < kFewDownWaves * S) break;
        if (S == 1 || us < least) { least = us; best = S; }
    }
    return best;
}
// the partial logits, and for more than kRouteTokens tokens the routing from them
static hipError_t launch_gate(const ExpertsArgs& a, hipStream_t stream) {
    const dim3 grid(gate_slices(a.d, a.N), ceil_div(a.T, kGateTokens));
    const auto go = [&](auto kern) { kern<<<grid, 256, 0, stream>>>(a.x, a.W_gate, a.T, a.d, a.N, const_cast<float*>(a.part)); };
    switch (gate_columns(a.N)) {
        case 8: go(&gate_part_kernel<8>); break;
        case 16: go(&gate_part_kernel<16>); break;
        case 32: go(&gate_part_kernel<32>); break;
        default: go(&gate_part_kernel<64>);
    }
    if (a.T > kRouteTokens) experts_route_kernel<<<ceil_div(a.T, 4), 256, 0, stream>>>(a);
    return hipGetLastError();
}

static int few_experts(const ExpertsArgs& a) { return a.T * a.k < a.N ? a.T * a.k : a.N; }   // in use, at most
// The kernels for up to 4 tokens, or those for more: in 4 bits up to 8 experts.  2 of 32 experts of 4096 and 1024 take 13.6 us with these and 23.4 with those, 8 take
// 21.8 and 28.7, 16 take 32.1 and 32.4; of 1024 and 1504 11.8 and 17.2, 20.2 and 20.5, 29.2 and 23.8.  In bf16 there is more to
// read in the same K tiles: 16 of 4096 and 1024 64.8 and 75.3, of 1024 and 1504 37.2 and 35.9.
template <typename WT>
static bool few_fits(const ExpertsArgs& a) {
    return a.T <= kFewTokens && a.T * few_row_bytes<WT>(a.d) <= kFewRowsMost && (!WT::kScales || few_experts(a) <= 8);
}

template <typename WT>
static hipError_t launch_few(const ExpertsArgs& a, hipStream_t stream) {
    constexpr int DD = kFewDownDepth<WT>, D2 = kFewDownDepth2<WT>;
    const int most = few_experts(a), rows = a.T * few_row_bytes<WT>(a.d), KS = few_up_split(most * ceil_div(a.f, 16), ceil_div(WT::row_bytes(a.d), 128));
    const auto up = [&](auto kern) {
        const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(kern), few_up_lds<WT>(kFewRowsMost, KS > 1));
        if (e != hipSuccess) return e;
        kern<<<kFewGroups, kFewWaves * 64, few_up_lds<WT>(rows, KS > 1), stream>>>(a);
        return hipGetLastError();
    };
    const hipError_t e = KS == 1 ? up(&experts_few_up_kernel<WT, 1>) : KS == 2 ? up(&experts_few_up_kernel<WT, 2>)
                       : KS == 4 ? up(&experts_few_up_kernel<WT, 4>) : up(&experts_few_up_kernel<WT, 8>);
    if (e != hipSuccess) return e;
    const int tiles = ceil_div(a.d, 16), splits = few_down_split<WT>(tiles, most, ceil_div(WT::row_bytes(a.f), 128));
    const auto down = [&](auto kern, int lds) {
        const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(kern), lds);
        if (e != hipSuccess) return e;
        kern<<<tiles * splits, kFewDownWaves * 64, lds, stream>>>(a, splits);
        return hipGetLastError();
    };
    const hipError_t f = tiles * splits <= 256 ? down(&experts_few_down_kernel<WT, kFewDownWaves, DD>, few_down_lds<WT, kFewDownWaves, DD>())
                                               : down(&experts_few_down_kernel<WT, kFewDownWaves, D2>, few_down_lds<WT, kFewDownWaves, D2>());
    if (f != hipSuccess) return f;
    if (splits > 1) experts_few_sum_kernel<<<ceil_div(a.T * a.d, 1024), 256, 0, stream>>>(a, splits);
    return hipGetLastError();
}
template <typename WT, int TB>
static hipError_t launch_many(const ExpertsArgs& a, hipStream_t stream) {
    constexpr int LDS = many_lds<WT, TB>();
    static_assert(LDS + (int)sizeof(Plan) + kExpertsMaxTokens * kMaxTopK <= 160 * 1024, "LDS");
    hipError_t e = start(&experts_many_kernel<WT, true, TB>, kManyGroups, kManyThreads, LDS, a, stream);
    if (e != hipSuccess) return e;
    e = start(&experts_many_kernel<WT, false, TB>, kManyGroups, kManyThreads, LDS, a, stream);
    if (e != hipSuccess) return e;
    experts_sum_kernel<<<dim3(ceil_div(a.d, 1024), a.T), 256, 0, stream>>>(a);
    return hipGetLastError();
}
template <typename WT>
static hipError_t launch(ExpertsArgs a, hipStream_t stream) {
    const bool few = few_fits<WT>(a);
    if (a.W_gate != nullptr && !(few && a.T == 1 && a.d * gate_columns(a.N) <= kGateHere)) {
        const hipError_t e = launch_gate(a, stream);
        if (e != hipSuccess) return e;
        a.W_gate = nullptr;   // done
    }
    if (few) return launch_few<WT>(a, stream);
    // Blocks of 16 or of 32 tokens, us.  4 bits: 64 tokens of 2 of 8 experts of 4096 and 3584 62.0 and 49.9, 32 tokens 43.6 and 48.6; 64 of 2 of 8 of 4096 and 14336
    // 174 and 150; 48 of 2 of 4 of 4096 41.3 and 38.5; 33 of 4 of 28 of 2080 and 1376 43.4 and 49.8; 64 of 2 of 64 of 1024 28.6 and 32.0.  bf16: 64 of 2 of 8 of 4096
    // and 3584 145 and 127, 32 tokens 127 and 127; 48 of 2 of 4 of 4096 and 2048 54.6 and 49.7; 20 of 2 of 16 of 4096 and 1024 78.5 and 78.2; 64 of 4 of 28 of 2048 and
    // 1024 75.9 and 76.1.
    return a.T * a.k <= 10 * a.N || a.T <= 16 ? launch_many<WT, 1>(a, stream) : launch_many<WT, 2>(a, stream);
}
hipError_t launch_experts(const ExpertsArgs& a, hipStream_t stream) {
    return a.s1 != nullptr ? launch<Mx4Weights>(a, stream) : launch<Bf16Weights>(a, stream);
}

size_t experts_h_bytes(int T, int k, int f) { return (size_t)T * k * f * sizeof(bf16_t); }
size_t experts_y_bytes(int T, int k, int d) { return (size_t)kManySplits * T * k * d * sizeof(float); }

size_t experts_part_bytes(int T, int d, int N) { return (size_t)T * gate_slices(d, N) * gate_columns(N) * sizeof(float); }

template <typename WT>
static hipError_t init_experts() {   // every kernel that launch_experts may start
    constexpr int DD = kFewDownDepth<WT>;
    hipError_t e = hipSuccess;
    const auto set = [&](const void* k, int lds) { if (e == hipSuccess) e = ensure_lds_limit(k, lds); };
    set(reinterpret_cast<const void*>(&experts_few_up_kernel<WT, 1>), few_up_lds<WT>(kFewRowsMost, false));
    set(reinterpret_cast<const void*>(&experts_few_up_kernel<WT, 2>), few_up_lds<WT>(kFewRowsMost, true));
    set(reinterpret_cast<const void*>(&experts_few_up_kernel<WT, 4>), few_up_lds<WT>(kFewRowsMost, true));
    set(reinterpret_cast<const void*>(&experts_few_up_kernel<WT, 8>), few_up_lds<WT>(kFewRowsMost, true));
    set(reinterpret_cast<const void*>(&experts_few_down_kernel<WT, kFewDownWaves, DD>), few_down_lds<WT, kFewDownWaves, DD>());
    set(reinterpret_cast<const void*>(&experts_few_down_kernel<WT, kFewDownWaves, kFewDownDepth2<WT>>), few_down_lds<WT, kFewDownWaves, kFewDownDepth2<WT>>());
    set(reinterpret_cast<const void*>(&experts_many_kernel<WT, true, 1>), many_lds<WT, 1>());
    set(reinterpret_cast<const void*>(&experts_many_kernel<WT, true, 2>), many_lds<WT, 2>());
    set(reinterpret_cast<const void*>(&experts_many_kernel<WT, false, 1>), many_lds<WT, 1>());
    set(reinterpret_cast<const void*>(&experts_many_kernel<WT, false, 2>), many_lds<WT, 2>());
    return e;
}
hipError_t experts_init_kernels() {
    const hipError_t e = init_experts<Bf16Weights>();
    return e != hipSuccess ? e : init_experts<Mx4Weights>();
}

}  // namespace meteora
