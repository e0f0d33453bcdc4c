// Gated MLPs of the experts that a few tokens (T <= 64) are routed to, and the gate in front of them:
//
//     h[t,j]  = silu(W1_e[0:f] x[t]) * (W1_e[f:2f] x[t]),    e = topk_idx[t,j],    silu(g) = g / (1 + exp(-g))
//     out[t]  = base[t] + scale * sum_j topk_w[t,j] * (W2_e h[t,j])
//
// Weights are bf16, or 4-bit values with block scales (quant_mx4.hpp) that become bf16 in registers, exactly, so that both run on
// v_mfma_f32_16x16x32_bf16 with x as it is: W is the first operand, the tokens are the 16 columns of the second.  h is rounded to bf16 once, as
// the operand of the second product; sums are fp32.
//
// The weights of the experts in use are what there is to read, once.  Every wavefront streams its rows of them through a ring of its own
// (see gemm_rows.hpp), K tiles of 128 bytes a row, with the tokens' rows beside them.  Which tokens an expert has every workgroup finds out
// for itself: a lane holds an expert's tokens as the bits of a word.  Two launches, and a third for more than 4 tokens:
//
// up to 4 tokens: the four columns are the tokens.  experts_few_up_kernel: 16 channels of h (32 rows of W1) to a wavefront, or to the
//   four of a workgroup, which split K then.  experts_few_down_kernel: 16 channels of the output to a workgroup, whose wavefronts split K and go
//   through the experts in use one after the other, so that the weighted sum is in registers and nothing is added in memory.
// more: an expert's tokens are columns, 16 or 32 at a time, read once for the four wavefronts of a workgroup, which have rows of W of
//   their own.  experts_up_kernel and experts_down_kernel; experts_sum_kernel adds the rows of a token.
#include <type_traits>

#include "common.hpp"
#include "gemm_mfma.hpp"
#include "gemm_rows.hpp"
#include "kernels.hpp"
#include "quant_mx4.hpp"
#include "topk_key.hpp"

namespace meteora {

constexpr int kFewTokens = 4;

// ---- routing: bit t of masks[e]: token t goes to expert e, by however many slots.  LDS; all threads of the workgroup.
struct ExpertMasks { uint32_t word[kMaxAdapters][2]; };

__device__ __forceinline__ void find_masks(const ExpertsArgs& a, ExpertMasks& m) {
    for (int i = threadIdx.x; i < 2 * kMaxAdapters; i += blockDim.x) m.word[i >> 1][i & 1] = 0;
    __syncthreads();
    for (int p = threadIdx.x; p < a.T * a.k; p += blockDim.x) {
        const int e = a.idx[p], t = p / a.k;
        if ((unsigned)e < (unsigned)a.N) atomicOr(&m.word[e][t >> 5], 1u << (t & 31));
    }
    __syncthreads();
}
__device__ __forceinline__ uint64_t mask_of(const ExpertMasks& m, int e) { return (uint64_t)m.word[e][1] << 32 | m.word[e][0]; }
__device__ __forceinline__ int rank_in(uint64_t mask, int t) { return __popcll(mask & (((uint64_t)1 << t) - 1)); }
// an inclusive sum over the lanes
__device__ __forceinline__ int wave_sums(int v, int lane) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int n = __shfl_up(v, off);
        if (lane >= off) v += n;
    }
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

// RB blocks of 16 rows of W in a wavefront's slots: the rows' bytes (see WaveOperand), then their words of scales
template <typename WT, int RB>
struct WeightRing {
    static constexpr int kLoads = RB * (2 + WT::kScales), kBytes = RB * WT::kBlockBytes;
    WaveOperand<RB> rows;
    ScaleRows scales;
    __amdgpu_buffer_rsrc_t scale_rsrc;
    uint32_t at_scale;
    // W: the first of `n` rows of `bytes` each; scale: that matrix's, with `all` rows, of which it is row0
    __device__ __forceinline__ WeightRing(const uint8_t* W, const uint8_t* scale, int all, int row0, int n, int bytes, int lane)
        : rows(reinterpret_cast<const int8_t*>(W), n, (uint32_t)bytes, lane), scales(scale, all, row0, n, bytes),
          at_scale((uint32_t)(lane & 15) * 16 + (lane >> 4) * 4) {}
    __device__ __forceinline__ void point(const uint8_t* W, const uint8_t* scale, int all, int row0, int n, int bytes) {
        rows.mat = i8_operand(reinterpret_cast<const int8_t*>(W), n, (uint32_t)bytes);
        scales = ScaleRows(scale, all, row0, n, bytes);
    }
    __device__ __forceinline__ void at_tile(int kt, int nk) {
        rows.at_tile(kt, nk);
        if constexpr (WT::kScales) scale_rsrc = scales.chunk(kt < nk ? kt >> 1 : scales.chunks);
    }
    __device__ __forceinline__ void request(unsigned char* slot) const {
#pragma unroll
        for (int j = 0; j < 2 * RB; ++j) rows.template request<kReadOnceI8>(slot, j);
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

template <typename WT, int KS, int D>
__global__ __launch_bounds__(256) void experts_few_up_kernel(const ExpertsArgs a) {
    constexpr int RB = 2, NL = FewTile<WT, RB>::kLoads, NP = FewTile<WT, RB>::kPieces, kSlot = few_slot_bytes<WT, RB>();
    constexpr int CH = 16 * (4 / KS);   // channels of a workgroup
    static_assert((D - 1) * NL < 64, "vmcnt");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ ExpertMasks masks;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, kq = lane >> 4;
    find_masks(a, masks);
    const uint64_t mine = lane < a.N ? mask_of(masks, lane) : 0;
    const uint64_t active = __ballot(mine != 0);
    const int tiles = ceil_div(a.f, CH), total = __popcll(active) * tiles;
    if ((int)blockIdx.x >= total) return;
    const int id = xcd_order(blockIdx.x, total);
    const int which = id / tiles;
    const int e = __builtin_amdgcn_readfirstlane(__ffsll(__ballot(mine != 0 && rank_in(active, lane) == which)) - 1);
    const int sums = wave_sums(__popcll(mine), lane);
    const int first = __builtin_amdgcn_readfirstlane(__shfl(sums, e) - __popcll(mask_of(masks, e)));   // row of h
    const uint32_t tokens = masks.word[e][0];
    const int c0 = (id - which * tiles) * CH + (KS == 1 ? wave * 16 : 0), n = min(16, a.f - c0);   // this wavefront's channels; n <= 0: none
    unsigned char* const ring = smem + wave * D * kSlot;

    const int bytes = WT::row_bytes(a.d), nk = ceil_div(bytes, 128), kp = KS == 1 ? 0 : wave;
    const int steps = n > 0 && kp < nk ? (nk - 1 - kp) / KS + 1 : 0;
    const uint8_t* W = a.W1 + ((size_t)e * 2 * a.f + c0) * bytes;
    const uint8_t* S = WT::kScales ? a.s1 + (size_t)e * mx4_scale_bytes(2 * a.f, a.d) : nullptr;
    WeightRing<WT, 1> g(W, S, 2 * a.f, c0, max(n, 0), bytes, lane), u(W + (size_t)a.f * bytes, S, 2 * a.f, a.f + c0, max(n, 0), bytes, lane);
    const auto x = token_rsrc(a.x, a.T, a.d);
    TokenPiece<WT> piece[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) piece[i].set(i * TokenPiece<WT>::kRows, lane);
#pragma unroll
    for (int i = 0; i < NP; ++i)
        piece[i].point(piece[i].row < kFewTokens && (tokens >> piece[i].row & 1) ? (uint32_t)piece[i].row * (uint32_t)a.d * 2u : kOutside);
    auto request = [&](unsigned char* slot, int kt) {
        const int end = n > 0 ? nk : 0;
        g.at_tile(kt, end);
        u.at_tile(kt, end);
        g.request(slot);
        u.request(slot + WT::kBlockBytes);
#pragma unroll
        for (int i = 0; i < NP; ++i)
            piece[i].request(x, slot + 2 * WT::kBlockBytes, i * TokenPiece<WT>::kRows, kt, end, (uint32_t)a.d * 2u);
    };
#pragma unroll
    for (int i = 0; i < D; ++i) request(ring + i * kSlot, kp + i * KS);
    f32x4 ag = {0.f, 0.f, 0.f, 0.f}, au = {0.f, 0.f, 0.f, 0.f};
    int at = 0;
    for (int s = 0; s < steps; ++s) {
        const int kt = kp + s * KS;
        unsigned char* const slot = ring + at * kSlot;
        at = at + 1 == D ? 0 : at + 1;
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * NL) : "memory");
        WeightFrags<WT, 1> wg, wu;
        wg.read(slot, kt, lane);
        wu.read(slot + WT::kBlockBytes, kt, lane);
        bf16x8 xf[WT::kSteps];
#pragma unroll
        for (int i = 0; i < WT::kSteps; ++i) xf[i] = token_frag<WT>(slot + 2 * WT::kBlockBytes, l15 & (kFewTokens - 1), kq, i);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slot is read
        request(slot, kt + D * KS);
#pragma unroll
        for (int i = 0; i < WT::kSteps; ++i) {
            ag = mfma_bf16(wg.at(i, 0), xf[i], ag);
            au = mfma_bf16(wu.at(i, 0), xf[i], au);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may land in what follows, or after the end
    if constexpr (KS > 1) {
        __syncthreads();
        f32x4* part = reinterpret_cast<f32x4*>(smem);
        part[wave * 128 + lane] = ag;
        part[wave * 128 + 64 + lane] = au;
        __syncthreads();
        if (wave != 0) return;
#pragma unroll
        for (int v = 1; v < KS; ++v) {
            ag += part[v * 128 + lane];
            au += part[v * 128 + 64 + lane];
        }
    }
    const int t = l15;
    if (t < kFewTokens && (tokens >> t & 1) && kq * 4 < n)   // f % 8 == 0
        store_h(a.h + (size_t)(first + rank_in(tokens, t)) * a.f + c0 + kq * 4, ag, au);
}

// The wavefronts split K (KS of them); sequence numbers run over the experts in use and their K tiles.
template <typename WT, int KS, int D>
__global__ __launch_bounds__(KS * 64) void experts_few_down_kernel(const ExpertsArgs a) {
    constexpr int NL = FewTile<WT, 1>::kLoads, NP = FewTile<WT, 1>::kPieces, kSlot = few_slot_bytes<WT, 1>();
    static_assert((D - 1) * NL < 64, "vmcnt");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ ExpertMasks masks;
    __shared__ int list[kMaxAdapters][2];                  // the experts in use and their first rows of h
    __shared__ float weight[kMaxAdapters][kFewTokens];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, kq = lane >> 4;
    find_masks(a, masks);
    const uint64_t mine = lane < a.N ? mask_of(masks, lane) : 0;
    const uint64_t active = __ballot(mine != 0);
    const int count = __popcll(active);
    if (wave == 0) {
        const int sums = wave_sums(__popcll(mine), lane);
        if (mine != 0) {
            const int i = rank_in(active, lane);
            list[i][0] = lane;
            list[i][1] = sums - __popcll(mine);
            for (int t = 0; t < kFewTokens; ++t) {
                float w = 0.f;
                for (int j = 0; j < a.k && t < a.T; ++j)
                    if (a.idx[t * a.k + j] == lane) w += a.w[t * a.k + j];
                weight[i][t] = w;
            }
        }
    }
    __syncthreads();
    const int c0 = xcd_order(blockIdx.x, gridDim.x) * 16, n = min(16, a.d - c0);
    unsigned char* const ring = smem + wave * D * kSlot;
    const int bytes = WT::row_bytes(a.f), nk = ceil_div(bytes, 128);
    const int per = wave < nk ? (nk - 1 - wave) / KS + 1 : 0, steps = per * count;
    const auto h = token_rsrc(a.h, a.T * a.k, a.f);
    WeightRing<WT, 1> w(a.W2, a.s2, a.d, c0, n, bytes, lane);
    TokenPiece<WT> piece[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) piece[i].set(i * TokenPiece<WT>::kRows, lane);
    int req_i = 0, req_kt = wave;   // next request: expert of the list, K tile
    auto point = [&](int i) {
        const int e = __builtin_amdgcn_readfirstlane(list[i][0]), row = __builtin_amdgcn_readfirstlane(list[i][1]);
        const uint32_t tokens = masks.word[e][0];
        w.point(a.W2 + ((size_t)e * a.d + c0) * bytes, WT::kScales ? a.s2 + (size_t)e * mx4_scale_bytes(a.d, a.f) : nullptr, a.d, c0, n, bytes);
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int t = piece[p].row;
            piece[p].point(t < kFewTokens && (tokens >> t & 1) ? (uint32_t)(row + rank_in(tokens, t)) * (uint32_t)a.f * 2u : kOutside);
        }
    };
    if (count > 0) point(0);
    auto request = [&](unsigned char* slot) {
        const int end = req_i < count && per > 0 ? nk : 0;
        w.at_tile(req_kt, end);
        w.request(slot);
#pragma unroll
        for (int p = 0; p < NP; ++p)
            piece[p].request(h, slot + WT::kBlockBytes, p * TokenPiece<WT>::kRows, req_kt, end, (uint32_t)a.f * 2u);
        req_kt += KS;
        if (req_kt >= nk && req_i < count) {
            req_kt = wave;
            if (++req_i < count) point(req_i);
        }
    };
#pragma unroll
    for (int i = 0; i < D; ++i) request(ring + i * kSlot);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f}, total = {0.f, 0.f, 0.f, 0.f};
    int at = 0, i = 0, kt = wave;
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
        if (kt >= nk) {   // the expert's last: its sum with the token's weight
            const int t = l15 & (kFewTokens - 1);
            const float wt = weight[i][t];
            const bool routed = masks.word[list[i][0]][0] >> t & 1;   // a column of zeros may meet a NaN in the weights
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                total[c] += routed ? wt * acc[c] : 0.f;
                acc[c] = 0.f;
            }
            kt = wave;
            ++i;
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may land in what follows
    __syncthreads();
    f32x4* part = reinterpret_cast<f32x4*>(smem);
    part[wave * 64 + lane] = total;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int v = 1; v < KS; ++v) total += part[v * 64 + lane];
    if (l15 >= a.T || l15 >= kFewTokens || kq * 4 >= n) return;
    const size_t o = (size_t)l15 * a.d + c0 + kq * 4;
    float v[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = a.scale * total[c] + (a.base != nullptr ? (float)a.base[o + c] : 0.f);
    *reinterpret_cast<uint2*>(a.out + o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

// ---- more tokens -----------------------------------------------------------------------------------------------------------------
// Blocks of R = 16 TB tokens of an expert, tiles of channels; the four wavefronts share the tokens' rows.
struct Block {
    int e, begin, count, first;   // expert, its tokens begin .. begin + count - 1, and the row of h and y of the first of these
};
template <int R>
struct Blocks {
    uint64_t mine;
    int sums, blocks, end, total;
    __device__ __forceinline__ Blocks(const ExpertsArgs& a, const ExpertMasks& m, int lane) {
        mine = lane < a.N ? mask_of(m, lane) : 0;
        sums = wave_sums(__popcll(mine), lane);
        blocks = (__popcll(mine) + R - 1) / R;
        end = wave_sums(blocks, lane);
        total = __builtin_amdgcn_readfirstlane(__shfl(end, 63));
    }
    __device__ __forceinline__ Block at(int b) const {
        const int e = __ffsll(__ballot(end > b)) - 1;
        const int n = __shfl(__popcll(mine), e), begin = (b - (__shfl(end, e) - __shfl(blocks, e))) * R;
        return {__builtin_amdgcn_readfirstlane(e), __builtin_amdgcn_readfirstlane(begin), __builtin_amdgcn_readfirstlane(min(R, n - begin)),
                __builtin_amdgcn_readfirstlane(__shfl(sums, e) - n + begin)};
    }
};

template <typename WT, int TB, int RB>
constexpr int many_slot_bytes() { return 4 * RB * WT::kBlockBytes + TB * 16 * kTokenBytes<WT>; }

// The loop over K of a workgroup: wavefront w has RB blocks of 16 rows, `rows` of them there are (by the ring), and the
// workgroup TB x 16 tokens, of which the first USED x 16 are multiplied.  `where(r)`: the first byte of token row r in `tokens`, or kOutside.
// USED is a constant, and a block of few tokens has a loop of its own: with a branch around the second 16 tokens' MFMAs the compiler moves
// accumulators behind the branch and leaves out the wait states for it (ROCm 7.2; tests/test_experts_host.py looks for that).
template <typename WT, int TB, int USED, int RB, int D, typename Ring, typename Where>
__device__ __forceinline__ void many_loop(f32x4 (&acc)[TB][RB], unsigned char* smem, Ring& ring, int nk, bool there, __amdgpu_buffer_rsrc_t tokens,
                                          uint32_t ld, int wave, int lane, Where where) {
    constexpr int kSlot = many_slot_bytes<WT, TB, RB>(), kRowsPer = TokenPiece<WT>::kRows, PIECES = TB * 16 / kRowsPer;
    constexpr int NP = PIECES < 4 ? 1 : PIECES / 4, NL = RB * (2 + WT::kScales) + NP;
    static_assert(D >= 3 && (D - 2) * NL < 64, "vmcnt");
    const int l15 = lane & 15, kq = lane >> 4;
    auto first_row = [&](int i) { return ((i * 4 + wave) % PIECES) * kRowsPer; };   // fewer than four pieces: some twice
    TokenPiece<WT> piece[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        piece[i].set(first_row(i), lane);
        piece[i].point(where(piece[i].row));
    }
    auto request = [&](int kt) {
        unsigned char* const slot = smem + kt % D * kSlot;
        ring.at_tile(kt, there ? nk : 0);
        ring.request(slot + wave * RB * WT::kBlockBytes);
#pragma unroll
        for (int i = 0; i < NP; ++i) piece[i].request(tokens, slot + 4 * RB * WT::kBlockBytes, first_row(i), kt, nk, ld);
    };
#pragma unroll
    for (int i = 0; i < D - 1; ++i) request(i);
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int r = 0; r < RB; ++r) acc[t][r] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int kt = 0; kt < nk; ++kt) {
        // this wavefront's part of the tile has landed, and so, behind the barrier, the others'; the slot before is read by all
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((D - 2) * NL) : "memory");
        request(kt + D - 1);
        const unsigned char* const slot = smem + kt % D * kSlot;
        WeightFrags<WT, RB> w;
        w.read(slot + wave * RB * WT::kBlockBytes, kt, lane);
        const unsigned char* const rows = slot + 4 * RB * WT::kBlockBytes;
#pragma unroll
        for (int i = 0; i < WT::kSteps; ++i) {
            bf16x8 wf[RB];
#pragma unroll
            for (int r = 0; r < RB; ++r) wf[r] = w.at(i, r);
#pragma unroll
            for (int t = 0; t < USED; ++t) {
                const bf16x8 xf = token_frag<WT>(rows, t * 16 + l15, kq, i);
#pragma unroll
                for (int r = 0; r < RB; ++r) acc[t][r] = mfma_bf16(wf[r], xf, acc[t][r]);
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// The rings of gate and up rows as one operand of two blocks
template <typename WT>
struct PairRing {
    WeightRing<WT, 1> g, u;
    __device__ __forceinline__ void at_tile(int kt, int nk) { g.at_tile(kt, nk); u.at_tile(kt, nk); }
    __device__ __forceinline__ void request(unsigned char* slot) const {   // as two blocks of one ring lie: rows, rows, scales, scales
#pragma unroll
        for (int j = 0; j < 2; ++j) g.rows.template request<kReadOnceI8>(slot, j);
#pragma unroll
        for (int j = 0; j < 2; ++j) u.rows.template request<kReadOnceI8>(slot + 2048, j);
        if constexpr (WT::kScales) {
            mx4_scale_lds(g.scale_rsrc, slot + 4096, g.at_scale);
            mx4_scale_lds(u.scale_rsrc, slot + 4352, u.at_scale);
        }
    }
};

template <typename WT, int TB, int D>
__global__ __launch_bounds__(256) void experts_up_kernel(const ExpertsArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ ExpertMasks masks;
    __shared__ int list[TB * 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, kq = lane >> 4;
    find_masks(a, masks);
    const Blocks<TB * 16> blocks(a, masks, lane);
    const int tiles = ceil_div(a.f, 64), total = blocks.total * tiles;
    if ((int)blockIdx.x >= total) return;
    const int id = xcd_order(blockIdx.x, total), column = id / blocks.total;
    const Block b = blocks.at(id - column * blocks.total);
    if (wave == 0) {
        const uint64_t m = mask_of(masks, b.e);
        const int r = rank_in(m, lane) - b.begin;
        if ((m >> lane & 1) && r >= 0 && r < b.count) list[r] = lane;
    }
    __syncthreads();
    const int c0 = column * 64 + wave * 16, n = min(16, a.f - c0);
    const int bytes = WT::row_bytes(a.d), nk = ceil_div(bytes, 128);
    const uint8_t* W = a.W1 + ((size_t)b.e * 2 * a.f + c0) * bytes;
    const uint8_t* S = WT::kScales ? a.s1 + (size_t)b.e * mx4_scale_bytes(2 * a.f, a.d) : nullptr;
    PairRing<WT> ring{WeightRing<WT, 1>(W, S, 2 * a.f, c0, max(n, 0), bytes, lane),
                      WeightRing<WT, 1>(W + (size_t)a.f * bytes, S, 2 * a.f, a.f + c0, max(n, 0), bytes, lane)};
    const auto tile = [&](auto used) __attribute__((always_inline)) {
        constexpr int USED = decltype(used)::value;
        f32x4 acc[TB][2];
        many_loop<WT, TB, USED, 2, D>(acc, smem, ring, nk, n > 0, token_rsrc(a.x, a.T, a.d), (uint32_t)a.d * 2u, wave, lane,
                                      [&](int r) { return r < b.count ? (uint32_t)list[r] * (uint32_t)a.d * 2u : kOutside; });
#pragma unroll
        for (int t = 0; t < USED; ++t)
            if (t * 16 + l15 < b.count && kq * 4 < n)
                store_h(a.h + (size_t)(b.first + t * 16 + l15) * a.f + c0 + kq * 4, acc[t][0], acc[t][1]);
    };
    if (TB == 1 || b.count <= 16) tile(std::integral_constant<int, 1>{});
    else tile(std::integral_constant<int, TB>{});
}

template <typename WT, int TB, int RB, int D>
__global__ __launch_bounds__(256) void experts_down_kernel(const ExpertsArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ ExpertMasks masks;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, kq = lane >> 4;
    find_masks(a, masks);
    const Blocks<TB * 16> blocks(a, masks, lane);
    const int tiles = ceil_div(a.d, 64 * RB), total = blocks.total * tiles;
    if ((int)blockIdx.x >= total) return;
    const int id = xcd_order(blockIdx.x, total), column = id / blocks.total;
    const Block b = blocks.at(id - column * blocks.total);
    const int c0 = (column * 4 + wave) * 16 * RB, n = min(16 * RB, a.d - c0);
    const int bytes = WT::row_bytes(a.f), nk = ceil_div(bytes, 128);
    WeightRing<WT, RB> ring(a.W2 + ((size_t)b.e * a.d + c0) * bytes, WT::kScales ? a.s2 + (size_t)b.e * mx4_scale_bytes(a.d, a.f) : nullptr, a.d,
                            c0, max(n, 0), bytes, lane);
    const auto tile = [&](auto used) __attribute__((always_inline)) {
        constexpr int USED = decltype(used)::value;
        f32x4 acc[TB][RB];
        many_loop<WT, TB, USED, RB, D>(acc, smem, ring, nk, n > 0, token_rsrc(a.h, a.T * a.k, a.f), (uint32_t)a.f * 2u, wave, lane,
                                       [&](int r) { return r < b.count ? (uint32_t)(b.first + r) * (uint32_t)a.f * 2u : kOutside; });
#pragma unroll
        for (int t = 0; t < USED; ++t)
#pragma unroll
            for (int r = 0; r < RB; ++r)
                if (t * 16 + l15 < b.count && r * 16 + kq * 4 < n)
                    *reinterpret_cast<f32x4*>(a.y + (size_t)(b.first + t * 16 + l15) * a.d + c0 + r * 16 + kq * 4) = acc[t][r];
    };
    if (TB == 1 || b.count <= 16) tile(std::integral_constant<int, 1>{});
    else tile(std::integral_constant<int, TB>{});
}

// out[t] = base[t] + scale * sum_j w[t,j] * y[row of (t, its expert j)], a token and 2048 channels to a workgroup
__global__ __launch_bounds__(256) void experts_sum_kernel(const ExpertsArgs a) {
    __shared__ ExpertMasks masks;
    const int tid = threadIdx.x, lane = tid & 63, t = blockIdx.y;
    find_masks(a, masks);
    const uint64_t mine = lane < a.N ? mask_of(masks, lane) : 0;
    const int row = wave_sums(__popcll(mine), lane) - __popcll(mine) + rank_in(mine, t);   // of this token for expert `lane`
    const int c = (blockIdx.x * 256 + tid) * 8;
    float sum[8] = {};
    for (int j = 0; j < a.k; ++j) {
        const int e = a.idx[t * a.k + j];
        if ((unsigned)e >= (unsigned)a.N) continue;
        const float w = a.w[t * a.k + j];
        const float* y = a.y + (size_t)__shfl(row, e) * a.d + c;
        if (c >= a.d) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += w * y[i];
    }
    if (c >= a.d) return;
    const size_t o = (size_t)t * a.d + c;
    uint32_t packed[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) v[h] = a.scale * sum[2 * i + h] + (a.base != nullptr ? (float)a.base[o + 2 * i + h] : 0.f);
        packed[i] = pack_bf16x2(v[0], v[1]);
    }
    *reinterpret_cast<u32x4*>(a.out + o) = u32x4{packed[0], packed[1], packed[2], packed[3]};
}

template <typename K>
static hipError_t start(K kern, int grid, int threads, int lds, const ExpertsArgs& a, hipStream_t stream) {
    const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(kern), lds);
    if (e != hipSuccess) return e;
    kern<<<grid, threads, lds, stream>>>(a);
    return hipGetLastError();
}
template <typename WT, int KS, int D>
constexpr int few_up_lds() { return 4 * D * few_slot_bytes<WT, 2>(); }
template <typename WT, int KS, int D>
constexpr int few_down_lds() { return KS * D * few_slot_bytes<WT, 1>(); }
template <typename WT, int TB, int RB, int D>
constexpr int many_lds() { return D * many_slot_bytes<WT, TB, RB>(); }
template <typename WT> constexpr int kFewUpDepth = WT::kScales ? 3 : 4;
template <typename WT> constexpr int kFewDownDepth = 5;

template <typename WT>
static hipError_t launch_few(const ExpertsArgs& a, hipStream_t stream) {
    constexpr int DU = kFewUpDepth<WT>, DD = kFewDownDepth<WT>;
    const int most = a.T * a.k < a.N ? a.T * a.k : a.N;   // experts in use
    const bool split = (int64_t)most * ceil_div(a.f, 64) < 256;
    const hipError_t e = split ? start(&experts_few_up_kernel<WT, 4, DU>, most * ceil_div(a.f, 16), 256, few_up_lds<WT, 4, DU>(), a, stream)
                               : start(&experts_few_up_kernel<WT, 1, DU>, most * ceil_div(a.f, 64), 256, few_up_lds<WT, 1, DU>(), a, stream);
    if (e != hipSuccess) return e;
    return start(&experts_few_down_kernel<WT, 4, DD>, ceil_div(a.d, 16), 256, few_down_lds<WT, 4, DD>(), a, stream);
}
template <typename WT, int TB>
static hipError_t launch_many(const ExpertsArgs& a, hipStream_t stream) {
    constexpr int D = WT::kScales && TB == 2 ? 4 : 3;
    const int most = a.T * a.k < a.N ? a.T * a.k : a.N;
    const int blocks = most + a.T * a.k / (16 * TB);   // sum of ceil(n_e / R) over the experts in use, sum of n_e <= T * k
    hipError_t e = start(&experts_up_kernel<WT, TB, D>, blocks * ceil_div(a.f, 64), 256, many_lds<WT, TB, 2, D>(), a, stream);
    if (e != hipSuccess) return e;
    e = start(&experts_down_kernel<WT, TB, 2, D>, blocks * ceil_div(a.d, 128), 256, many_lds<WT, TB, 2, D>(), a, stream);
    if (e != hipSuccess) return e;
    experts_sum_kernel<<<dim3(ceil_div(a.d, 2048), a.T), 256, 0, stream>>>(a);
    return hipGetLastError();
}
template <typename WT>
static hipError_t launch(const ExpertsArgs& a, hipStream_t stream) {
    if (a.T <= kFewTokens) return launch_few<WT>(a, stream);
    return a.T <= 16 ? launch_many<WT, 1>(a, stream) : launch_many<WT, 2>(a, stream);
}
hipError_t launch_experts(const ExpertsArgs& a, hipStream_t stream) {
    return a.s1 != nullptr ? launch<Mx4Weights>(a, stream) : launch<Bf16Weights>(a, stream);
}

size_t experts_h_bytes(int T, int k, int f) { return (size_t)T * k * f * sizeof(bf16_t); }
size_t experts_y_bytes(int T, int k, int d) { return T <= kFewTokens ? 0 : (size_t)T * k * d * sizeof(float); }

// ---- the gate of a few tokens: a token to a workgroup, logits[j] = sum_i x[i] W_gate[i,j] + bias[j], top-k and softmax ------------
// Lanes hold columns of W_gate, 64 / NP rows a load instruction; fp32 sums in a fixed order.
template <int NP>
__global__ __launch_bounds__(1024) void gate_few_kernel(const bf16_t* __restrict__ x, const float* __restrict__ W_gate,
                                                        const float* __restrict__ bias, int d, int N, int k, float inv_temperature,
                                                        int32_t* __restrict__ topk_idx, float* __restrict__ topk_w) {
    constexpr int SUB = 64 / NP, STEP = 16 * SUB, U = 8;
    __shared__ float part[16][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane % NP, t = blockIdx.x;
    const bf16_t* row = x + (size_t)t * d;
    float sum[2] = {0.f, 0.f};
    for (int i0 = wave * SUB + lane / NP; i0 < d; i0 += STEP * U) {
        float w[U], v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * STEP;
            const bool in = i < d && col < N;
            w[u] = in ? W_gate[(size_t)i * N + col] : 0.f;
            v[u] = in ? (float)row[i] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) sum[u & 1] = fmaf(v[u], w[u], sum[u & 1]);
    }
    float s = sum[0] + sum[1];
#pragma unroll
    for (int off = NP; off < 64; off <<= 1) s += __shfl_xor(s, off);
    part[wave][lane] = s;
    __syncthreads();
    if (wave != 0) return;
    float g[1] = {0.f};
    if (lane < N) {
        const int at = lane % NP;
#pragma unroll
        for (int v = 0; v < 16; ++v) g[0] += part[v][at];
        g[0] += bias != nullptr ? bias[lane] : 0.f;
        if (g[0] == 0.f) g[0] = 0.f;   // -0 -> +0 so equal logits have equal keys
    }
    int sel[1];
    float w[1];
    wave_topk_softmax<64, 1>(g, lane, N, k, inv_temperature, sel, w);
    if (lane < k) {
        topk_idx[(size_t)t * k + lane] = sel[0];
        topk_w[(size_t)t * k + lane] = w[0];
    }
}
hipError_t launch_gate_few(const void* x, const float* W_gate, const float* bias, int T, int d, int N, int k, float inv_temperature,
                           int32_t* topk_idx, float* topk_w, hipStream_t stream) {
    const auto go = [&](auto kern) {
        kern<<<T, 1024, 0, stream>>>((const bf16_t*)x, W_gate, bias, d, N, k, inv_temperature, topk_idx, topk_w);
        return hipGetLastError();
    };
    return N <= 8 ? go(&gate_few_kernel<8>) : N <= 16 ? go(&gate_few_kernel<16>) : N <= 32 ? go(&gate_few_kernel<32>) : go(&gate_few_kernel<64>);
}

template <typename WT>
static hipError_t init_experts() {   // every kernel that launch_experts may start
    constexpr int DU = kFewUpDepth<WT>, DD = kFewDownDepth<WT>, D2 = WT::kScales ? 4 : 3;
    hipError_t e = hipSuccess;
    const auto set = [&](const void* k, int lds) { if (e == hipSuccess) e = ensure_lds_limit(k, lds); };
    set(reinterpret_cast<const void*>(&experts_few_up_kernel<WT, 4, DU>), few_up_lds<WT, 4, DU>());
    set(reinterpret_cast<const void*>(&experts_few_up_kernel<WT, 1, DU>), few_up_lds<WT, 1, DU>());
    set(reinterpret_cast<const void*>(&experts_few_down_kernel<WT, 4, DD>), few_down_lds<WT, 4, DD>());
    set(reinterpret_cast<const void*>(&experts_up_kernel<WT, 1, 3>), many_lds<WT, 1, 2, 3>());
    set(reinterpret_cast<const void*>(&experts_up_kernel<WT, 2, D2>), many_lds<WT, 2, 2, D2>());
    set(reinterpret_cast<const void*>(&experts_down_kernel<WT, 1, 2, 3>), many_lds<WT, 1, 2, 3>());
    set(reinterpret_cast<const void*>(&experts_down_kernel<WT, 2, 2, D2>), many_lds<WT, 2, 2, D2>());
    return e;
}
hipError_t experts_init_kernels() {
    const hipError_t e = init_experts<Bf16Weights>();
    return e != hipSuccess ? e : init_experts<Mx4Weights>();
}

}  // namespace meteora
