// What the products of rows over groups of consecutive rows have in common, whatever a row's bytes stand for (8-bit integers,
// 4-bit values with block scales): the tiles of the groups, the operands of the wavefronts' rings, and the choice of a tile.
#pragma once
#include <math.h>

#include "common.hpp"
#include "gemm_mfma.hpp"
#include "kernels.hpp"

namespace meteora {

constexpr int kI8Tile = 128;   // bytes of a K tile, and what 64 bf16 inputs are in the bf16 kernels

template <typename S>
struct GemmRowsArgs {
    const int8_t* q;        // [T, d_in]
    const S* q_scale;       // of the type's own layout
    const int8_t* W;        // [N, d_out, d_in]
    const S* w_scale;
    const int32_t* offsets; // [N+1], or nullptr: one group of all rows
    void* out;              // [T, d_out]
    int T, d_in, d_out, N;  // d_in: bytes of a row
    int tiles_m, tiles_n;   // row tiles of the grid (at least as many as there are), column tiles
    int tile_cols;          // columns of a tile (wave kernel)
    int tail;               // 1: the tiles of a last, half-empty round are left to the product's tail kernel (gemm_i8_, gemm_mx4_tail_kernel)
    int past_caches;        // 1: W is more than the caches keep from one call to the next
};

// The row tiles of all groups, each cut into tiles of BM rows, one group behind the other.  Whatever the offsets hold, the rows lie in
// [0, T).  A lane holds a group; uniform results.
struct RowTile {
    int e, row0, rows;
    bool alone;   // its group has no other
};

template <int BM>
struct RowTiles {
    int lo, hi, mine, end;   // this lane's group: its rows, its tiles, and those up to its last
    int count;               // of all groups
    template <typename Args>
    __device__ __forceinline__ RowTiles(const Args& a, int lane) {
        if (a.offsets == nullptr) {
            count = a.tiles_m;
            return;
        }
        lo = hi = 0;
        if (lane < a.N) {
            lo = min(max(a.offsets[lane], 0), a.T);
            hi = min(max(a.offsets[lane + 1], lo), a.T);
        }
        mine = end = (hi - lo + BM - 1) / BM;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int n = __shfl_up(end, off);
            if (lane >= off) end += n;
        }
        count = min(__builtin_amdgcn_readfirstlane(__shfl(end, 63)), a.tiles_m);
    }
    template <typename Args>
    __device__ __forceinline__ RowTile at(const Args& a, int tile) const {   // tile < count
        if (a.offsets == nullptr) return {0, tile * BM, min(BM, a.T - tile * BM), count == 1};
        const int e = __ffsll(__ballot(end > tile)) - 1;
        const int first = __shfl(lo, e) + (tile - (__shfl(end, e) - __shfl(mine, e))) * BM;
        const int rows = min(BM, __shfl(hi, e) - first);
        return {__builtin_amdgcn_readfirstlane(e), __builtin_amdgcn_readfirstlane(first), __builtin_amdgcn_readfirstlane(rows),
                __builtin_amdgcn_readfirstlane(__shfl(mine, e)) == 1};
    }
};
// The grid's row tiles: as many as T rows in N groups can make.  Workgroups past those that there are end at once.
template <typename Args>
static int most_row_tiles(const Args& a, int BM) {
    const int64_t most = (int64_t)ceil_div(a.T, BM) + (a.offsets != nullptr ? a.N - 1 : 0);
    return (int)(most < a.T ? most : a.T);
}

// Columns of a tile of up to `most` where the tiles do not fill the CUs: as many tiles as there are CUs, in whole eights.
static int wave_tile_cols(int row_tiles, int d_out, int most) {
    if ((int64_t)row_tiles * ceil_div(d_out, most) > 256 || most == 16) return most;
    return ceil_div(ceil_div(d_out, 256 / row_tiles), 8) * 8;
}

// The workgroups of an XCD take consecutive tiles (ids are dealt to the 8 XCDs in turn), row tiles of the same columns of W
// next to each other.
__device__ __forceinline__ int xcd_order(int wg, int total) {
    const int per = total / 8, rest = total % 8, xcd = wg % 8;
    return xcd * per + min(xcd, rest) + wg / 8;
}

// Cache policy of the weights of few rows: "nt", for weights that come from memory, as a model's layers in turn do; what it costs where they
// are still in a cache, or where many row tiles read long rows again, is accepted.  Read once and kept, us, weights in turn: 8 groups of
// 4096 -> 4096, 16 rows 25.8 and 29.0, 16 x 4096 -> 4096 5.7 and 6.0, 64 x 4096 -> 4096 7.9 and 8.2, 16 x 5120 -> 13824 13.7 and 15.2, 64 x
// 14336 -> 4096 22.8 and 22.1, 64 and 700 x 131056 -> 264 106 and 79, 215 and 146; the same weights again and again: 26.9 and 23.8, 4.0
// and 4.0, 5.8 and 5.8, 12.9 and 12.9, 21.2 and 13.5, 110 and 59, 216 and 134.
constexpr int kReadOnceI8 = 2;
constexpr uint32_t kOutside = 0x80000000u;   // past every resource here, also with a K offset added

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

struct I8Operand { __amdgpu_buffer_rsrc_t rsrc; };
__device__ __forceinline__ I8Operand i8_operand(const int8_t* base, int rows, uint32_t ld) {
    return {__builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(base), 0, (uint32_t)rows * ld, 0x00020000)};
}

template <int POLICY>
__device__ __forceinline__ void i8_load_lds(const I8Operand& o, unsigned char* dst, uint32_t voff, int soff) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(o.rsrc, (__attribute__((address_space(3))) void*)dst, 16, voff, soff, 0, POLICY);
}

// One operand of the wavefront rings: an instruction moves 8 rows x 128 bytes; 16-byte chunk c of row r lies at position swz(r, c).
// Rows past the last load zeros, as do a last K tile's columns past d_in.  Requests may go on past the last K tile, from behind the
// matrix's end, so that their number is always the same.
template <int B>
struct WaveOperand {
    I8Operand mat;
    uint32_t even, odd, even_last, odd_last, ld8;   // offsets of the chunk in rows j * 8 + (lane / 8), j even and odd
    uint32_t v_even, v_odd, kbase;
    int last;                                       // the K tile that is partly there
    __device__ __forceinline__ WaveOperand(const int8_t* base, int rows, uint32_t ld, int lane) : mat(i8_operand(base, rows, ld)) {
        const int rsub = lane >> 3, p = lane & 7;
        const uint32_t c_even = (uint32_t)swz(rsub, p) * 16, c_odd = (uint32_t)swz(rsub + 8, p) * 16, left = ld % 128;
        even = (uint32_t)rsub * ld + c_even;
        odd = (uint32_t)rsub * ld + c_odd;
        even_last = c_even < left ? even : kOutside;
        odd_last = c_odd < left ? odd : kOutside;
        ld8 = ld * 8;
        last = left != 0 ? (int)(ld / 128) : -1;
    }
    __device__ __forceinline__ void at_tile(int kt, int nk) {
        v_even = kt == last ? even_last : even;
        v_odd = kt == last ? odd_last : odd;
        kbase = kt < nk ? (uint32_t)kt * 128 : kOutside;
    }
    template <int POLICY>
    __device__ __forceinline__ void request(unsigned char* slot, int j) const {   // rows j * 8 to j * 8 + 7 of the K tile
        i8_load_lds<POLICY>(mat, slot + j * 1024, j & 1 ? v_odd : v_even, (int)(kbase + (uint32_t)j * ld8));
    }
};

// 256 x 256 tiles, one to a CU, beyond whole rounds of 256 of them: up to 128 are done in smaller tiles, one or two to a CU, by a second
// launch instead of as a round of their own.  The first of them:
constexpr int kTailTiles = 128;
__host__ __device__ constexpr int tail_start(int tiles) {
    return tiles > 256 && tiles % 256 <= kTailTiles ? tiles - tiles % 256 : tiles;
}

constexpr int kTailSmall = 16, kTailMiddle = 32;   // tiles of 256 x 256 that are 256 of 64 x 64, and of 128 x 64
template <typename Args>
static bool may_have_tail(const Args& a, int64_t tiles) {   // the most that there may be, of 256 x 256
    return tiles > 256 && (a.offsets != nullptr || tail_start((int)tiles) != tiles);
}

// The shapes of the tiles that there are, and the fitted times of each, see the products.
struct I8Shape {
    int rows, cols, per_cu;
    bool wave;              // gemm_i8_wave_kernel
    float launch, round, step, share;
};
constexpr int kI8ShapeCount = 13;

template <typename Args>
static float shape_us(const Args& a, const I8Shape (&shapes)[kI8ShapeCount], const I8Shape& s, float row_tiles, int cols, float groups) {   // groups: with rows
    const float nk = (float)ceil_div(a.d_in, kI8Tile), tiles = row_tiles * (float)ceil_div(a.d_out, cols);
    float rounds = ceilf(tiles / (float)(256 * s.per_cu)), tail = 0.f;
    const float rest = tiles - 256.f * (rounds - 1.f);
    if (s.rows * s.cols == 256 * 256 && rounds > 1.f && rest <= (float)kTailTiles) {
        const I8Shape& q = shapes[rest <= (float)kTailSmall ? 4 : rest <= (float)kTailMiddle ? 6 : 8];   // much the same rings
        rounds -= 1.f;
        tail = q.launch + q.round + nk * q.step + rest * (float)(256 * 256 / (q.rows * q.cols)) / 256.f * nk * q.share;
    }
    const float own = s.launch + rounds * (s.round + nk * s.step) + (tail > 0.f ? rounds : tiles / 256.f) * nk * s.share + tail;
    const float mem = (groups * (float)a.d_out * (float)a.d_in + (float)a.T * ((float)a.d_in + 2.f * (float)a.d_out)) / (s.wave ? 5.1e6f : 4.9e6f);
    return cbrtf(own * own * own + mem * mem * mem);
}

// Rows of the groups of one deal, as far as tiles of 16 rows or more tell them apart
struct Deal {
    float groups = 0.f, weight = 1.f;   // with rows; each value below stands for `weight` groups
    float small = 0.f;                  // of them with up to 16 rows
    int n = 0, rows[kMaxAdapters];
    void add(int r) {
        if (r <= 0) return;
        groups += weight;
        if (r <= 16) small += weight;
        else rows[n++] = r;
    }
    float tiles(int tile_rows) const {
        int t = 0;
        for (int i = 0; i < n; ++i) t += ceil_div(rows[i], tile_rows);
        return small + weight * (float)t;
    }
};

template <typename Args>
static int choose_shape(const Args& a, const I8Shape (&shapes)[kI8ShapeCount]) {
    const bool grouped = a.offsets != nullptr && a.N > 1;
    Deal even, falling;
    if (grouped) {
        const int N = a.T < a.N ? a.T : a.N;
        const float mean = (float)a.T / (float)N, spread = 1.22f * sqrtf(mean);
        even.weight = (float)N / 3.f;
        for (int i = -1; i <= 1; ++i) even.add((int)(mean + (float)i * spread + 0.5f));
        float sum = 0.f;
        for (int j = 1; j <= N; ++j) sum += 1.f / (float)(j * j);
        for (int j = 1; j <= N; ++j) falling.add((int)((float)a.T / (sum * (float)(j * j)) + 0.5f));
    }
    int best = 0;
    float least = 0.f;
    for (int i = 0; i < kI8ShapeCount; ++i) {
        const I8Shape& s = shapes[i];
        const int cols = s.wave ? wave_tile_cols(most_row_tiles(a, s.rows), a.d_out, s.cols) : s.cols;
        const float us = !grouped ? shape_us(a, shapes, s, (float)ceil_div(a.T, s.rows), cols, 1.f)
                                  : shape_us(a, shapes, s, even.tiles(s.rows), cols, even.groups) +
                                        shape_us(a, shapes, s, falling.tiles(s.rows), cols, falling.groups);
        if (i == 0 || us < least) { least = us; best = i; }
    }
    return best;
}

}  // namespace meteora
