// Rows next to each other by adapter, and back (Sec. 3.3: the token sets X_i of the adapters, here as rows that are moved).
//
//   sort      pos[t,j] = the place of pair (t, j) among all pairs with an id in [0, N), in order of adapter, then token, then
//             slot; -1 for other ids.  Row pos[t,j] of xs is x[t], as it is or as 8-bit whole numbers (quant.hpp).
//   unsort    out[t] = base[t] + scale * sum_j w[t,j] * ys[pos[t,j]]; with w = 1 the gradient of sort.
//   backward  of unsort: dys[pos[t,j]] = scale * w[t,j] * dy[t],  dw[t,j] = scale * <dy[t], ys[pos[t,j]]>.
//
// All of them move bytes and nothing else, so every one goes by tokens: a token's row is read once and written k times, or k
// rows are read and one written, at places that pos names; nothing is added to memory, and results do not depend on an order.
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"
#include "quant.hpp"

namespace meteora {

constexpr int kSortThreads = 256;

// ---- positions ------------------------------------------------------------------------------------------------------------
// How often each adapter stands in a list of ids, counted by a workgroup in LDS.  8 copies of every counter, a lane's own by its low
// bits, so that a skewed load does not make 64 lanes wait for one word.  Counts: the order does not show.
constexpr int kCopies = 8, kCopyStride = kCopies + 1;   // copies of one counter lie in different banks
struct Counters { int n[kMaxAdapters * kCopyStride]; };
__device__ __forceinline__ void clear(Counters& c) {
    for (int i = threadIdx.x; i < kMaxAdapters * kCopyStride; i += kSortThreads) c.n[i] = 0;
}
__device__ __forceinline__ void count(Counters& c, int key, int by) {
    atomicAdd(&c.n[key * kCopyStride + (threadIdx.x & (kCopies - 1))], by);
}
__device__ __forceinline__ int total(const Counters& c, int key) {
    int sum = 0;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) sum += c.n[key * kCopyStride + i];
    return sum;
}

// chunk_counts[c][j] = pairs of chunk c with id j
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const int32_t* __restrict__ topk_idx, int64_t pairs,
                                                                  int chunk_pairs, int N, int32_t* __restrict__ chunk_counts) {
    __shared__ Counters c;
    clear(c);
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * chunk_pairs;
    for (int i = threadIdx.x; i < chunk_pairs && base + i < pairs; i += kSortThreads) {
        const int key = topk_idx[base + i];
        if (key >= 0 && key < N) count(c, key, 1);
    }
    __syncthreads();
    if (threadIdx.x < N) chunk_counts[(size_t)blockIdx.x * N + threadIdx.x] = total(c, threadIdx.x);
}

struct SortArgs {
    const int32_t* topk_idx;
    int64_t pairs;                 // T * k
    int T, k, N, d, chunk_tokens, nchunks;
    const int32_t* chunk_counts;   // of sort_count_kernel, or nullptr: every workgroup counts all ids
    int32_t* pos;                  // [T,k]
    int32_t* offsets;              // [N+1]
    float* xs_scale;               // [T*k]
};

// The one-launch form: every workgroup counts all pairs, so it takes few of them and up to 1024 workgroups.  ceil(T / 1024) tokens to a
// workgroup, T * k <= kOneLaunchPairs: at most T * k / 1024 + k pairs.
constexpr int kOneLaunchPairs = 16384, kOneLaunchChunks = 1024;
constexpr int kSortChunkPairs = kOneLaunchPairs / kOneLaunchChunks + kMaxTopK;

struct SortShared {
    Counters before, rest;
    int running[kMaxAdapters], wave_hist[2][4][kMaxAdapters];   // of the even and the odd steps: a step's is read into the next one
};

// The same for up to 256 pairs in all (decode), without a table: every wavefront holds all ids, and a place is the number of pairs
// with a smaller id or the same and an earlier place in line, counted by ballots.  64 tokens x 4096, top-2: 4.6 us, with tables 6.0.
constexpr int kFewPairs = 256;
__device__ __forceinline__ void sort_few_positions(const SortArgs& a, int* places) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), pairs = (int)a.pairs;
    int id[kFewPairs / 64];
#pragma unroll
    for (int u = 0; u < kFewPairs / 64; ++u) {
        const int v = u * 64 + lane < pairs ? a.topk_idx[u * 64 + lane] : -1;
        id[u] = v >= 0 && v < a.N ? v : a.N;   // behind all
    }
    auto smaller = [&](int key) {
        int n = 0;
#pragma unroll
        for (int u = 0; u < kFewPairs / 64; ++u) n += __popcll(__ballot(id[u] < key));
        return n;
    };
    const int chunk_pairs = a.chunk_tokens * a.k, base = blockIdx.x * chunk_pairs;
    for (int i = wave; i < chunk_pairs && base + i < pairs; i += kSortThreads / 64) {
        const int p = base + i, key = a.topk_idx[p];
        int place = -1;
        if (key >= 0 && key < a.N) {
            place = smaller(key);
#pragma unroll
            for (int u = 0; u < kFewPairs / 64; ++u) place += __popcll(__ballot(id[u] == key && u * 64 + lane < p));
        }
        if (lane == 0) {
            places[i] = place;
            a.pos[p] = place;
        }
    }
    if (blockIdx.x == 0)
        for (int e = wave; e <= a.N; e += kSortThreads / 64) {
            const int first = smaller(e);   // e = N: all that are below it
            if (lane == 0) a.offsets[e] = first;
        }
    __syncthreads();
}

// The places of this workgroup's chunk of pairs, to pos and, if there is, to LDS.
__device__ __forceinline__ void sort_positions(const SortArgs& a, SortShared& sh, int* places) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x;
    const int chunk_pairs = a.chunk_tokens * a.k;
    const int64_t base = (int64_t)c * chunk_pairs;
    auto key_at = [&](int i) { return i < chunk_pairs && base + i < a.pairs ? a.topk_idx[base + i] : -1; };
    int next_key = key_at(threadIdx.x);   // on its way while the ids are counted
    clear(sh.before);
    clear(sh.rest);
    __syncthreads();
    if (a.chunk_counts == nullptr) {
        // 16 ids a thread at a time, all requested before the first is counted: the loop waits for loads, not for arithmetic
        const int pairs = (int)a.pairs, first = (int)base;
        for (int i0 = threadIdx.x * 4; i0 < pairs; i0 += kSortThreads * 16) {
            int4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * kSortThreads * 4;
                v[u] = make_int4(-1, -1, -1, -1);
                if (i + 4 <= pairs) v[u] = *reinterpret_cast<const int4*>(a.topk_idx + i);
                else if (i < pairs) v[u] = make_int4(a.topk_idx[i], i + 1 < pairs ? a.topk_idx[i + 1] : -1, i + 2 < pairs ? a.topk_idx[i + 2] : -1, -1);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * kSortThreads * 4;
                const int key[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (key[e] >= 0 && key[e] < a.N) count(i + e < first ? sh.before : sh.rest, key[e], 1);
            }
        }
    } else {
        const int entries = a.nchunks * a.N, first = c * a.N;
        for (int i0 = threadIdx.x; i0 < entries; i0 += kSortThreads * 8) {
            int n[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) n[u] = i0 + u * kSortThreads < entries ? a.chunk_counts[i0 + u * kSortThreads] : 0;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int i = i0 + u * kSortThreads;
                if (n[u] != 0) count(i < first ? sh.before : sh.rest, i % a.N, n[u]);
            }
        }
    }
    __syncthreads();
    if (wave == 0) {
        const int b = total(sh.before, lane), v = b + total(sh.rest, lane);   // adapters from N on: zeros
        int incl = v;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int n = __shfl_up(incl, off);
            if (lane >= off) incl += n;
        }
        sh.running[lane] = incl - v + b;
        if (c == 0) {
            if (lane < a.N) a.offsets[lane] = incl - v;
            if (lane == a.N - 1) a.offsets[a.N] = incl;
        }
    }
    for (int i0 = 0; i0 < chunk_pairs; i0 += kSortThreads) {
        const int i = i0 + threadIdx.x;
        const bool in = i < chunk_pairs && base + i < a.pairs;
        const int key = next_key;
        next_key = key_at(i + kSortThreads);
        const bool valid = key >= 0 && key < a.N;
        unsigned long long peers = __ballot(valid);   // lanes of this wavefront with the same id
#pragma unroll
        for (int bit = 0; bit < 6; ++bit) {
            const unsigned long long m = __ballot(valid && ((key >> bit) & 1));
            peers &= ((key >> bit) & 1) ? m : ~m;
        }
        const int rank = __popcll(peers & (lane == 0 ? 0ull : ~0ull >> (64 - lane)));
        auto& hist = sh.wave_hist[i0 / kSortThreads & 1];
        hist[wave][lane] = 0;
        __syncthreads();
        if (valid && rank == 0) hist[wave][key] = __popcll(peers);
        __syncthreads();
        int p = -1;
        if (valid) {
            p = sh.running[key] + rank;
            for (int w = 0; w < wave; ++w) p += hist[w][key];
        }
        if (in) {
            if (places != nullptr) places[i] = p;
            a.pos[base + i] = p;
        }
        __syncthreads();
        if (i0 + kSortThreads < chunk_pairs && threadIdx.x < kMaxAdapters)
            sh.running[threadIdx.x] += hist[0][threadIdx.x] + hist[1][threadIdx.x] + hist[2][threadIdx.x] + hist[3][threadIdx.x];
    }
    __syncthreads();
}

// Many pairs: the places alone, and the rows in a launch of their own.
__global__ __launch_bounds__(kSortThreads) void sort_places_kernel(const SortArgs a) {
    __shared__ SortShared sh;
    sort_positions(a, sh, nullptr);
}

__global__ __launch_bounds__(kSortThreads) void sort_move_kernel(const SortArgs a, const u32x4* __restrict__ x, int row16,
                                                                 int lanes_log2, u32x4* __restrict__ xs) {
    const int t = (int)((blockIdx.x * (int64_t)kSortThreads + threadIdx.x) >> lanes_log2);
    if (t >= a.T) return;
    const int lanes = 1 << lanes_log2;
    for (int i = threadIdx.x & (lanes - 1); i < row16; i += lanes) {
        const u32x4 v = x[(size_t)t * row16 + i];
        for (int j = 0; j < a.k; ++j) {
            const int p = a.pos[(size_t)t * a.k + j];
            if (p >= 0) xs[(size_t)p * row16 + i] = v;
        }
    }
}

template <typename TX, int G, int HELD>
__global__ __launch_bounds__(kSortThreads) void sort_move_quantize_kernel(const SortArgs a, const TX* __restrict__ x,
                                                                          int8_t* __restrict__ xs) {
    __shared__ float red[4];
    const int t = (int)((blockIdx.x * (unsigned)kSortThreads + threadIdx.x) / G);
    if (t >= a.T) return;   // G = 256: never
    const TX* src = x + (size_t)t * a.d;
    const int32_t* place = a.pos + (size_t)t * a.k;
    QuantRow<TX, G, HELD> r;
    r.load(src, a.d / 8);
    const float top = r.top(src, a.d / 8, red);
    r.store(src, a.d / 8, top, [&](int i, uint2 v) {
        for (int j = 0; j < a.k; ++j)
            if (place[j] >= 0) reinterpret_cast<uint2*>(xs + (size_t)place[j] * a.d)[i] = v;
    });
    const int lane = threadIdx.x & (G - 1);
    if (lane < a.k && place[lane] >= 0) a.xs_scale[place[lane]] = top / 127.f;
}

// Rows as they are, 16 bytes a piece; 2^lanes_log2 threads to a row.  The first pieces are on their way while the places are found.
constexpr int kSortHeld = 8;
__global__ __launch_bounds__(kSortThreads) void sort_rows_kernel(const SortArgs a, const u32x4* __restrict__ x, int row16,
                                                                 int lanes_log2, u32x4* __restrict__ xs) {
    __shared__ SortShared sh;
    __shared__ int places[kSortChunkPairs];
    const int t0 = blockIdx.x * a.chunk_tokens, tokens = min(a.chunk_tokens, a.T - t0);
    const int lanes = 1 << lanes_log2, lane = threadIdx.x & (lanes - 1);
    struct Cursor { int t, c; };
    Cursor get{(int)threadIdx.x >> lanes_log2, lane}, put = get;
    if (lane >= row16) get.t = put.t = tokens;
    auto next = [&](Cursor& p) {
        p.c += lanes;
        if (p.c >= row16) {
            p.c = lane;
            p.t += kSortThreads >> lanes_log2;
        }
    };
    u32x4 held[kSortHeld];
    auto load = [&] {
#pragma unroll
        for (int u = 0; u < kSortHeld; ++u) {
            if (get.t < tokens) held[u] = x[(size_t)(t0 + get.t) * row16 + get.c];
            next(get);
        }
    };
    load();
    if (a.pairs <= kFewPairs) sort_few_positions(a, places);
    else sort_positions(a, sh, places);
    while (put.t < tokens) {
#pragma unroll
        for (int u = 0; u < kSortHeld; ++u) {
            if (put.t < tokens)
                for (int j = 0; j < a.k; ++j) {
                    const int p = places[put.t * a.k + j];
                    if (p >= 0) xs[(size_t)p * row16 + put.c] = held[u];
                }
            next(put);
        }
        load();
    }
}

// Rows as 8-bit whole numbers
template <typename TX, int G, int HELD>
__global__ __launch_bounds__(kSortThreads) void sort_quantize_kernel(const SortArgs a, const TX* __restrict__ x,
                                                                     int8_t* __restrict__ xs) {
    static_assert(kSortThreads == kQuantThreads, "a workgroup quantises a row");
    __shared__ SortShared sh;
    __shared__ int places[kSortChunkPairs];
    __shared__ float red[2][4];
    const int t0 = blockIdx.x * a.chunk_tokens, tokens = min(a.chunk_tokens, a.T - t0), pieces = a.d / 8;
    const TX* rows = x + (size_t)t0 * a.d;
    constexpr int GROUPS = kSortThreads / G;
    QuantRow<TX, G, HELD> r;
    int t = threadIdx.x / G;
    if (t < tokens) r.load(rows + (size_t)t * a.d, pieces);
    if (a.pairs <= kFewPairs) sort_few_positions(a, places);
    else sort_positions(a, sh, places);
    for (int n = 0; t < tokens; t += GROUPS, ++n) {   // G = 256: the same for all threads
        const TX* src = rows + (size_t)t * a.d;
        const int* place = places + t * a.k;
        const float top = r.top(src, pieces, red[n & 1]);
        r.store(src, pieces, top, [&](int i, uint2 v) {
            for (int j = 0; j < a.k; ++j)
                if (place[j] >= 0) reinterpret_cast<uint2*>(xs + (size_t)place[j] * a.d)[i] = v;
        });
        const int lane = threadIdx.x & (G - 1);
        if (lane < a.k && place[lane] >= 0) a.xs_scale[place[lane]] = top / 127.f;
        if (t + GROUPS < tokens) r.load(src + (size_t)GROUPS * a.d, pieces);
    }
}

// One launch or three, whole calls of top-2 unless said, as they are / quantised: 2001 x 4096 12.7 and 15.4 / 13.1 and 16.0 us, 4096 x
// 4096 20.2 and 28.9 / 23.6 and 25.6, 8192 x 4096 40.4 and 43.0 / 42.6 and 35.6, 8192 x 1024 16.3 and 18.5 / 16.8 and 18.5; top-8 2048 x
// 1024 14.7 and 21.0 / 15.1 and 22.2, 4096 x 1024 31.8 and 22.0 / 31.1 and 20.2 (as 256 workgroups 20.7 / 22.2).
static bool sort_in_one(int64_t pairs, int64_t elements, bool quantised) {
    return pairs <= kOneLaunchPairs && !(quantised && elements > (int64_t)1 << 24);
}
static int sort_chunk_tokens(int T) { return ceil_div(T, kOneLaunchChunks); }
// With many, a launch of histograms, one of places, which adds up those of all chunks, and one of rows.
constexpr int kCountChunks = 256;
static int count_chunk_tokens(int T) { return ceil_div(T, kCountChunks); }
size_t sort_count_bytes(int N) { return (size_t)kCountChunks * N * sizeof(int32_t); }

// threads to a row, as a power of two: at most a workgroup's
static int lanes_log2_for(int row16) {
    int l = 0;
    while (l < 8 && (1 << l) < row16) ++l;
    return l;
}

template <typename TX>
static hipError_t launch_sort_quantize(const SortArgs& a, const TX* x, int8_t* xs, hipStream_t stream) {
    return quant_row_shape(a.d, a.chunk_tokens >= 4, [&](auto g, auto held) {
        sort_quantize_kernel<TX, decltype(g)::value, decltype(held)::value><<<a.nchunks, kSortThreads, 0, stream>>>(a, x, xs);
        return hipGetLastError();
    });
}

template <typename TX>
static hipError_t launch_move_quantize(const SortArgs& a, const TX* x, int8_t* xs, hipStream_t stream) {
    return quant_row_shape(a.d, a.T >= 2048, [&](auto g, auto held) {
        constexpr int G = decltype(g)::value, HELD = decltype(held)::value;
        sort_move_quantize_kernel<TX, G, HELD><<<ceil_div(a.T, kSortThreads / G), kSortThreads, 0, stream>>>(a, x, xs);
        return hipGetLastError();
    });
}

hipError_t launch_sort_tokens(const void* x, const int32_t* topk_idx, int T, int k, int N, int d, bool bf16, void* xs,
                              float* xs_scale, int32_t* pos, int32_t* offsets, int32_t* chunk_counts, hipStream_t stream) {
    SortArgs a{};
    a.topk_idx = topk_idx; a.pairs = (int64_t)T * k; a.T = T; a.k = k; a.N = N; a.d = d;
    a.pos = pos; a.offsets = offsets; a.xs_scale = xs_scale;
    const int row16 = d / (bf16 ? 8 : 4), lanes = lanes_log2_for(row16);
    if (sort_in_one(a.pairs, (int64_t)T * d, xs_scale != nullptr)) {
        a.chunk_tokens = sort_chunk_tokens(T);
        if (a.chunk_tokens * k > kSortChunkPairs) return hipErrorInvalidValue;   // places[] of the kernels
        a.nchunks = ceil_div(T, a.chunk_tokens);
        if (xs_scale != nullptr)
            return bf16 ? launch_sort_quantize(a, (const bf16_t*)x, (int8_t*)xs, stream)
                        : launch_sort_quantize(a, (const float*)x, (int8_t*)xs, stream);
        sort_rows_kernel<<<a.nchunks, kSortThreads, 0, stream>>>(a, (const u32x4*)x, row16, lanes, (u32x4*)xs);
        return hipGetLastError();
    }
    a.chunk_tokens = count_chunk_tokens(T);
    a.nchunks = ceil_div(T, a.chunk_tokens);
    a.chunk_counts = chunk_counts;
    sort_count_kernel<<<a.nchunks, kSortThreads, 0, stream>>>(topk_idx, a.pairs, a.chunk_tokens * k, N, chunk_counts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    sort_places_kernel<<<a.nchunks, kSortThreads, 0, stream>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (xs_scale != nullptr)
        return bf16 ? launch_move_quantize(a, (const bf16_t*)x, (int8_t*)xs, stream)
                    : launch_move_quantize(a, (const float*)x, (int8_t*)xs, stream);
    sort_move_kernel<<<(unsigned)ceil_div64((int64_t)T << lanes, kSortThreads), kSortThreads, 0, stream>>>(a, (const u32x4*)x, row16, lanes,
                                                                                                 (u32x4*)xs);
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
    int blocks;           // 0, or workgroups that share it, a piece to a thread
    float scale;
};

template <typename TX>
__global__ __launch_bounds__(256) void unsort_kernel(const UnsortArgs a, const u32x4* __restrict__ ys,
                                                     const u32x4* base, u32x4* out) {   // base may be out
    int t, i, step;
    if (a.blocks > 0) {
        t = blockIdx.x / a.blocks;
        i = (blockIdx.x - t * a.blocks) * 256 + threadIdx.x;
        step = a.row16;
    } else {
        t = (int)((blockIdx.x * 256ll + threadIdx.x) >> a.lanes_log2);
        step = 1 << a.lanes_log2;
        i = threadIdx.x & (step - 1);
    }
    if (t >= a.T) return;
    for (; i < a.row16; i += step) {
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

hipError_t launch_unsort_tokens(const void* ys, int64_t rows, const int32_t* pos, const float* w, int T, int k, int d, bool bf16,
                                float scale, const void* base, void* out, hipStream_t stream) {
    UnsortArgs a{pos, w, T, k, d / (bf16 ? 8 : 4), rows, 0, 0, scale};
    a.lanes_log2 = lanes_log2_for(a.row16);
    // A piece to a thread, unless that is more threads than a launch has (2^32): a loop over the pieces of a row waits for memory once
    // per step.  Loop and piece, top-2: 64 x 4096 4.4 and 3.7 us, 64 x 14336 10.6 and 4.5, 4096 x 4096 25.0 and 23.5.
    if (a.row16 >= 256 && (int64_t)T * ceil_div(a.row16, 256) < (int64_t)1 << 24) a.blocks = ceil_div(a.row16, 256);
    const unsigned grid = a.blocks > 0 ? (unsigned)(T * a.blocks) : (unsigned)ceil_div64((int64_t)T << a.lanes_log2, 256);
    if (bf16) unsort_kernel<bf16_t><<<grid, 256, 0, stream>>>(a, (const u32x4*)ys, (const u32x4*)base, (u32x4*)out);
    else unsort_kernel<float><<<grid, 256, 0, stream>>>(a, (const u32x4*)ys, (const u32x4*)base, (u32x4*)out);
    return hipGetLastError();
}

// One workgroup, or 2^lanes_log2 of its threads, per token.  THREADS: 256, and for few tokens with long rows 1024, so that the loop over a
// row waits for memory fewer times.
template <typename TX, int THREADS>
__global__ __launch_bounds__(THREADS) void unsort_backward_kernel(const UnsortArgs a, const u32x4* __restrict__ dy,
                                                                  const u32x4* __restrict__ ys, u32x4* __restrict__ dys,
                                                                  float* __restrict__ dw) {
    __shared__ float part[THREADS / 64][kMaxTopK];
    const int t = (int)((blockIdx.x * (int64_t)THREADS + threadIdx.x) >> a.lanes_log2);
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
    const int wave = threadIdx.x >> 6, per = lanes / 64;   // wavefronts that share a token
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
    UnsortArgs a{pos, w, T, k, d / (bf16 ? 8 : 4), rows, 0, 0, scale};
    a.lanes_log2 = lanes_log2_for(a.row16);
    auto go = [&](auto kern, int threads) {
        kern<<<(unsigned)ceil_div64((int64_t)T << a.lanes_log2, threads), threads, 0, stream>>>(a, (const u32x4*)dy, (const u32x4*)ys,
                                                                                               (u32x4*)dys, dw);
        return hipGetLastError();
    };
    // 256 threads to a row and 1024, us, top-2: 64 x 4096 7.4 and 6.4, 64 x 14336 14.8 and 9.0, 512 x 4096 12.0 and 10.4, 512 x 14336 25.4 and
    // 19.3, 640 x 4096 13.1 and 16.1, 640 x 8192 19.9 and 20.6, 520 x 14336 25.8 and 24.7, 768 x 14336 31.6 and 31.2, 1024 x 14336 36.0 and
    // 37.0; top-8 300 x 5120 36.2 and 21.4, 640 x 5120 43.7 and 38.0, 640 x 14336 99.7 and 81.6: the border is that of top-2
    if (a.row16 >= 512 && T <= 512) {
        a.lanes_log2 = 10;
        return bf16 ? go(&unsort_backward_kernel<bf16_t, 1024>, 1024) : go(&unsort_backward_kernel<float, 1024>, 1024);
    }
    return bf16 ? go(&unsort_backward_kernel<bf16_t, 256>, 256) : go(&unsort_backward_kernel<float, 256>, 256);
}

}  // namespace meteora
