// Rows next to each other by adapter, and back (Sec. 3.3: the token sets X_i of the adapters, here as rows that are moved).
//
//   sort      pos[t,j] = the place of pair (t, j) among all pairs with an id in [0, N), in order of adapter, then token, then
//             slot; -1 for other ids.  Row pos[t,j] of xs is x[t], as it is or as 8-bit whole numbers (quant.hpp).
//   unsort    out[t] = base[t] + scale * sum_j w[t,j] * ys[pos[t,j]]; with w = 1 the gradient of sort.
//   backward  of unsort: dys[pos[t,j]] = scale * w[t,j] * dy[t],  dw[t,j] = scale * <dy[t], ys[pos[t,j]]>.
//
// All of them move bytes and nothing else, so every one goes by tokens: a token's row is read once and written k times, or k
// rows are read and one written, at places that pos names; nothing is added to memory, and results do not depend on an order.
#include "common.hpp"
#include "kernels.hpp"
#include "quant.hpp"

namespace meteora {

constexpr int kSortThreads = 256;

// ---- positions ------------------------------------------------------------------------------------------------------------
// chunk_counts[c][j] = pairs of chunk c (chunk_tokens tokens) with id j
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const int32_t* __restrict__ topk_idx, int64_t pairs,
                                                                  int chunk_pairs, int N, int32_t* __restrict__ chunk_counts) {
    __shared__ int hist[kMaxAdapters];
    if (threadIdx.x < kMaxAdapters) hist[threadIdx.x] = 0;
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * chunk_pairs;
    for (int i = threadIdx.x; i < chunk_pairs && base + i < pairs; i += kSortThreads) {
        const int key = topk_idx[base + i];
        if (key >= 0 && key < N) atomicAdd(&hist[key], 1);   // counts: the order does not show
    }
    __syncthreads();
    if (threadIdx.x < N) chunk_counts[(size_t)blockIdx.x * N + threadIdx.x] = hist[threadIdx.x];
}

struct SortArgs {
    const int32_t* topk_idx;
    int64_t pairs;                 // T * k
    int T, k, N, d, chunk_tokens, nchunks;
    const int32_t* chunk_counts;
    int32_t* pos;                  // [T,k]
    int32_t* offsets;              // [N+1]
    float* xs_scale;               // [T*k]
};

// A workgroup's chunk of tokens: the first place of every adapter's pairs of this chunk, then the chunk's pairs in order.
__device__ __forceinline__ void sort_positions(const SortArgs& a, int* places /*LDS, chunk pairs*/) {
    __shared__ int tot[4][kMaxAdapters], bef[4][kMaxAdapters], running[kMaxAdapters], wave_hist[4][kMaxAdapters];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x;
    int t = 0, b = 0;
    if (lane < a.N)
        for (int cc = wave; cc < a.nchunks; cc += 4) {
            const int v = a.chunk_counts[(size_t)cc * a.N + lane];
            t += v;
            if (cc < c) b += v;
        }
    tot[wave][lane] = t;
    bef[wave][lane] = b;
    __syncthreads();
    if (wave == 0) {
        const int v = tot[0][lane] + tot[1][lane] + tot[2][lane] + tot[3][lane];
        int incl = v;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int n = __shfl_up(incl, off);
            if (lane >= off) incl += n;
        }
        running[lane] = incl - v + bef[0][lane] + bef[1][lane] + bef[2][lane] + bef[3][lane];
        if (c == 0) {
            if (lane < a.N) a.offsets[lane] = incl - v;
            if (lane == a.N - 1) a.offsets[a.N] = incl;
        }
    }
    __syncthreads();
    const int chunk_pairs = a.chunk_tokens * a.k;
    const int64_t base = (int64_t)c * chunk_pairs;
    for (int i0 = 0; i0 < chunk_pairs; i0 += kSortThreads) {
        const int i = i0 + threadIdx.x;
        const bool in = i < chunk_pairs && base + i < a.pairs;
        const int key = in ? a.topk_idx[base + i] : -1;
        const bool valid = key >= 0 && key < a.N;
        unsigned long long peers = __ballot(valid);   // lanes of this wavefront with the same id
#pragma unroll
        for (int bit = 0; bit < 6; ++bit) {
            const unsigned long long m = __ballot(valid && ((key >> bit) & 1));
            peers &= ((key >> bit) & 1) ? m : ~m;
        }
        const int rank = __popcll(peers & (lane == 0 ? 0ull : ~0ull >> (64 - lane)));
        wave_hist[wave][lane] = 0;
        __syncthreads();
        if (valid && rank == 0) wave_hist[wave][key] = __popcll(peers);
        __syncthreads();
        int p = -1;
        if (valid) {
            p = running[key] + rank;
            for (int w = 0; w < wave; ++w) p += wave_hist[w][key];
        }
        if (in) {
            places[i] = p;
            a.pos[base + i] = p;
        }
        __syncthreads();
        if (threadIdx.x < kMaxAdapters)
            running[threadIdx.x] += wave_hist[0][threadIdx.x] + wave_hist[1][threadIdx.x] + wave_hist[2][threadIdx.x] +
                                    wave_hist[3][threadIdx.x];
        __syncthreads();
    }
}

constexpr int kSortChunkPairs = 2048;   // at most, in LDS

// rows as they are, 16 bytes a piece
__global__ __launch_bounds__(kSortThreads) void sort_rows_kernel(const SortArgs a, const u32x4* __restrict__ x, int row16,
                                                                 u32x4* __restrict__ xs) {
    __shared__ int places[kSortChunkPairs];
    sort_positions(a, places);
    const int t0 = blockIdx.x * a.chunk_tokens, tokens = min(a.chunk_tokens, a.T - t0);
    for (int t = 0; t < tokens; ++t)
        for (int i = threadIdx.x; i < row16; i += kSortThreads) {
            const u32x4 v = x[(size_t)(t0 + t) * row16 + i];
            for (int j = 0; j < a.k; ++j) {
                const int p = places[t * a.k + j];
                if (p >= 0) xs[(size_t)p * row16 + i] = v;
            }
        }
}

// rows as 8-bit whole numbers
template <typename TX, int HELD>
__global__ __launch_bounds__(kSortThreads) void sort_quantize_kernel(const SortArgs a, const TX* __restrict__ x,
                                                                     int8_t* __restrict__ xs) {
    static_assert(kSortThreads == kQuantThreads, "a workgroup quantises a row");
    __shared__ int places[kSortChunkPairs];
    __shared__ float red[2][4];
    sort_positions(a, places);
    const int t0 = blockIdx.x * a.chunk_tokens, tokens = min(a.chunk_tokens, a.T - t0);
    for (int t = 0; t < tokens; ++t) {
        const int* place = places + t * a.k;
        const float top = quantize_row<TX, HELD>(x + (size_t)(t0 + t) * a.d, a.d / 8, red[t & 1], [&](int i, uint2 v) {
            for (int j = 0; j < a.k; ++j)
                if (place[j] >= 0) reinterpret_cast<uint2*>(xs + (size_t)place[j] * a.d)[i] = v;
        });
        if ((int)threadIdx.x < a.k && place[threadIdx.x] >= 0) a.xs_scale[place[threadIdx.x]] = top / 127.f;
    }
}

// Tokens per workgroup: the histograms of all chunks are read by every workgroup.
constexpr int kSortChunks = 512;
static int sort_chunk_tokens(int T, int k) {
    int c = 1;
    while (c < kSortChunkPairs / k / 2 && ceil_div(T, c) > kSortChunks) c *= 2;
    return c;
}
size_t sort_count_bytes(int T, int k, int N) { return (size_t)ceil_div(T, sort_chunk_tokens(T, k)) * N * sizeof(int32_t); }
size_t sort_count_bytes_reserved(int T, int k, int N) {   // of any batch of up to T tokens
    const size_t few = (size_t)(T < kSortChunks ? T : kSortChunks) * N * sizeof(int32_t), own = sort_count_bytes(T, k, N);
    return own > few ? own : few;
}

template <typename TX>
static hipError_t launch_sort_quantize(const SortArgs& a, const TX* x, int8_t* xs, hipStream_t stream) {
    const int per_thread = ceil_div(a.d / 8, kQuantThreads);
    auto go = [&](auto kern) {
        kern<<<a.nchunks, kSortThreads, 0, stream>>>(a, x, xs);
        return hipGetLastError();
    };
    if (per_thread <= 1) return go(&sort_quantize_kernel<TX, 1>);
    if (per_thread <= 2) return go(&sort_quantize_kernel<TX, 2>);
    if (per_thread <= 4) return go(&sort_quantize_kernel<TX, 4>);
    if (per_thread <= kQuantHeld) return go(&sort_quantize_kernel<TX, kQuantHeld>);
    return go(&sort_quantize_kernel<TX, 0>);
}

hipError_t launch_sort_tokens(const void* x, const int32_t* topk_idx, int T, int k, int N, int d, bool bf16, void* xs,
                              float* xs_scale, int32_t* pos, int32_t* offsets, int32_t* chunk_counts, hipStream_t stream) {
    SortArgs a{};
    a.topk_idx = topk_idx; a.pairs = (int64_t)T * k; a.T = T; a.k = k; a.N = N; a.d = d;
    a.chunk_tokens = sort_chunk_tokens(T, k); a.nchunks = ceil_div(T, a.chunk_tokens);
    a.chunk_counts = chunk_counts; a.pos = pos; a.offsets = offsets; a.xs_scale = xs_scale;
    sort_count_kernel<<<a.nchunks, kSortThreads, 0, stream>>>(topk_idx, a.pairs, a.chunk_tokens * k, N, chunk_counts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (xs_scale != nullptr)
        return bf16 ? launch_sort_quantize(a, (const bf16_t*)x, (int8_t*)xs, stream)
                    : launch_sort_quantize(a, (const float*)x, (int8_t*)xs, stream);
    sort_rows_kernel<<<a.nchunks, kSortThreads, 0, stream>>>(a, (const u32x4*)x, d / (bf16 ? 8 : 4), (u32x4*)xs);
    return hipGetLastError();
}

// ---- back -----------------------------------------------------------------------------------------------------------------
// 16 bytes of a row as fp32
template <typename TX> struct Piece16;
template <> struct Piece16<bf16_t> {
    static constexpr int kN = 8;
    static __device__ __forceinline__ void get(const u32x4& v, float (&f)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(v[i] << 16);
            f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ u32x4 put(const float (&f)[8]) {
        return u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
    }
};
template <> struct Piece16<float> {
    static constexpr int kN = 4;
    static __device__ __forceinline__ void get(const u32x4& v, float (&f)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
    }
    static __device__ __forceinline__ u32x4 put(const float (&f)[4]) {
        return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
};

struct UnsortArgs {
    const int32_t* pos;   // [T,k]
    const float* w;       // [T,k] or nullptr: ones
    int T, k, row16;
    int64_t rows;         // of ys: places are below it
    int lanes_log2;       // threads that share a token's row
    float scale;
};

template <typename TX>
__global__ __launch_bounds__(256) void unsort_kernel(const UnsortArgs a, const u32x4* __restrict__ ys,
                                                     const u32x4* base, u32x4* out) {   // base may be out
    const int t = (int)((blockIdx.x * 256ll + threadIdx.x) >> a.lanes_log2);
    if (t >= a.T) return;
    const int lanes = 1 << a.lanes_log2;
    for (int i = threadIdx.x & (lanes - 1); i < a.row16; i += lanes) {
        constexpr int n = Piece16<TX>::kN;
        float sum[n] = {}, f[n];
        for (int j = 0; j < a.k; ++j) {
            const int p = a.pos[(size_t)t * a.k + j];
            if (p < 0 || p >= a.rows) continue;
            const float w = a.w ? a.w[(size_t)t * a.k + j] : 1.f;
            Piece16<TX>::get(ys[(size_t)p * a.row16 + i], f);
#pragma unroll
            for (int e = 0; e < n; ++e) sum[e] += w * f[e];
        }
        if (base != nullptr) {
            Piece16<TX>::get(base[(size_t)t * a.row16 + i], f);
#pragma unroll
            for (int e = 0; e < n; ++e) f[e] += a.scale * sum[e];
        } else {
#pragma unroll
            for (int e = 0; e < n; ++e) f[e] = a.scale * sum[e];
        }
        out[(size_t)t * a.row16 + i] = Piece16<TX>::put(f);
    }
}

static int lanes_log2_for(int row16) {
    int l = 0;
    while (l < 8 && (1 << l) < row16) ++l;
    return l;
}

hipError_t launch_unsort_tokens(const void* ys, int64_t rows, const int32_t* pos, const float* w, int T, int k, int d, bool bf16,
                                float scale, const void* base, void* out, hipStream_t stream) {
    UnsortArgs a{pos, w, T, k, d / (bf16 ? 8 : 4), rows, 0, scale};
    a.lanes_log2 = lanes_log2_for(a.row16);
    const unsigned grid = (unsigned)ceil_div64((int64_t)T << a.lanes_log2, 256);
    if (bf16) unsort_kernel<bf16_t><<<grid, 256, 0, stream>>>(a, (const u32x4*)ys, (const u32x4*)base, (u32x4*)out);
    else unsort_kernel<float><<<grid, 256, 0, stream>>>(a, (const u32x4*)ys, (const u32x4*)base, (u32x4*)out);
    return hipGetLastError();
}

// One workgroup, or 2^lanes_log2 of its threads, per token.
template <typename TX>
__global__ __launch_bounds__(256) void unsort_backward_kernel(const UnsortArgs a, const u32x4* __restrict__ dy,
                                                              const u32x4* __restrict__ ys, u32x4* __restrict__ dys,
                                                              float* __restrict__ dw) {
    __shared__ float part[4][kMaxTopK];
    const int t = (int)((blockIdx.x * 256ll + threadIdx.x) >> a.lanes_log2);
    const int lanes = 1 << a.lanes_log2;
    float dot[kMaxTopK] = {};
    if (t < a.T)
        for (int i = threadIdx.x & (lanes - 1); i < a.row16; i += lanes) {
            constexpr int n = Piece16<TX>::kN;
            float g[n], f[n];
            Piece16<TX>::get(dy[(size_t)t * a.row16 + i], g);
#pragma unroll
            for (int j = 0; j < kMaxTopK; ++j) {
                if (j >= a.k) break;
                const int p = a.pos[(size_t)t * a.k + j];
                if (p < 0 || p >= a.rows) continue;
                const float sw = a.scale * (a.w ? a.w[(size_t)t * a.k + j] : 1.f);
                if (dw != nullptr) {
                    Piece16<TX>::get(ys[(size_t)p * a.row16 + i], f);
#pragma unroll
                    for (int e = 0; e < n; ++e) dot[j] += g[e] * f[e];
                }
#pragma unroll
                for (int e = 0; e < n; ++e) f[e] = sw * g[e];
                dys[(size_t)p * a.row16 + i] = Piece16<TX>::put(f);
            }
        }
    if (dw == nullptr) return;
#pragma unroll
    for (int j = 0; j < kMaxTopK; ++j)
        for (int off = min(lanes, 64) >> 1; off >= 1; off >>= 1) dot[j] += __shfl_xor(dot[j], off);
    if (lanes <= 64) {
        if (t < a.T && (threadIdx.x & (lanes - 1)) == 0)
#pragma unroll
            for (int j = 0; j < kMaxTopK; ++j)
                if (j < a.k) dw[(size_t)t * a.k + j] = a.scale * dot[j];
        return;
    }
    const int wave = threadIdx.x >> 6, per = lanes / 64;   // 2 or 4 wavefronts share a token
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int j = 0; j < kMaxTopK; ++j) part[wave][j] = dot[j];
    __syncthreads();
    const int in = threadIdx.x & (lanes - 1);
    if (t < a.T && in < a.k) {
        float sum = 0.f;
        for (int v = 0; v < per; ++v) sum += part[wave + v][in];
        dw[(size_t)t * a.k + in] = a.scale * sum;
    }
}

hipError_t launch_unsort_backward(const void* dy, const void* ys, int64_t rows, const int32_t* pos, const float* w, int T, int k,
                                  int d, bool bf16, float scale, void* dys, float* dw, hipStream_t stream) {
    UnsortArgs a{pos, w, T, k, d / (bf16 ? 8 : 4), rows, 0, scale};
    a.lanes_log2 = lanes_log2_for(a.row16);
    const unsigned grid = (unsigned)ceil_div64((int64_t)T << a.lanes_log2, 256);
    if (bf16) unsort_backward_kernel<bf16_t><<<grid, 256, 0, stream>>>(a, (const u32x4*)dy, (const u32x4*)ys, (u32x4*)dys, dw);
    else unsort_backward_kernel<float><<<grid, 256, 0, stream>>>(a, (const u32x4*)dy, (const u32x4*)ys, (u32x4*)dys, dw);
    return hipGetLastError();
}

}  // namespace meteora
