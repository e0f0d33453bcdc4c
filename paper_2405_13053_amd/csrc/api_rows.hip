// Entry points of the 8-bit products and of the rows sorted by adapter (declared in include/meteora.h): argument validation and
// the launch sequence of each.  No device memory is allocated here and nothing synchronises with the host.
#include <math.h>

#include "../../include/meteora.h"
#include "common.hpp"
#include "kernels.hpp"

using namespace meteora;

namespace {

constexpr int kI8MaxInputs = 131056;   // 128 * 128 of each add up to less than 2^31
constexpr int kI8MaxOutputs = 1 << 20;
constexpr int kRowsMax = (1 << 24) - 1;   // a launch has fewer than 2^32 threads, up to 256 to a row

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool known(meteora_dtype dt) { return dt == METEORA_F32 || dt == METEORA_BF16; }
inline meteora_status status(hipError_t e) { return e == hipSuccess ? METEORA_OK : METEORA_ERR_HIP; }

bool sort_shape_ok(int T, int k, int N) { return T >= 0 && k >= 1 && N >= 1; }
bool sort_shape_supported(int T, int k, int N) {
    return N <= kMaxAdapters && k <= kMaxTopK && T <= kRowsMax;   // T * k < 2^31
}
size_t base_gemm_i8_bytes(int T, int d_in) {   // the quantised rows, then their scales
    return align_up((size_t)T * d_in, 256) + align_up((size_t)T * sizeof(float), 256);
}

}  // namespace

extern "C" {

meteora_status meteora_quantize_rows(const void* x, int rows, int d, meteora_dtype dt, int8_t* q, float* scale,
                                     meteora_stream stream) {
    if (!x || !q || !scale || rows < 0 || d < 1) return METEORA_ERR_INVALID_ARG;
    if (!known(dt) || d % 8 != 0 || rows > kRowsMax || !aligned(x, 16) || !aligned(q, 16) || !aligned(scale, 16))
        return METEORA_ERR_UNSUPPORTED;
    if (rows == 0) return METEORA_OK;
    return status(launch_quantize_rows(x, rows, d, dt == METEORA_BF16, q, scale, static_cast<hipStream_t>(stream)));
}

static bool i8_sizes_supported(int T, int d_in, int d_out) {
    return d_in % 16 == 0 && d_in <= kI8MaxInputs && d_out % 8 == 0 && d_out <= kI8MaxOutputs && T <= kRowsMax &&
           (int64_t)T * d_out < (int64_t)1 << 33;
}

static meteora_status check_i8_weights(const int8_t* W, const float* w_scale, int T, int d_in, int d_out, meteora_dtype dt,
                                       const void* out) {
    if (!W || !w_scale || !out || T < 0 || d_in < 1 || d_out < 1) return METEORA_ERR_INVALID_ARG;
    if (!known(dt) || !i8_sizes_supported(T, d_in, d_out)) return METEORA_ERR_UNSUPPORTED;
    if (!aligned(W, 16) || !aligned(w_scale, 16) || !aligned(out, 16)) return METEORA_ERR_UNSUPPORTED;
    return METEORA_OK;
}

meteora_status meteora_gemm_i8(const int8_t* q, const float* q_scale, const int8_t* W, const float* w_scale,
                               const int32_t* offsets, int T, int d_in, int d_out, int N, meteora_dtype dt, void* out,
                               meteora_stream stream) {
    if (!q || !q_scale || N < 1 || (offsets == nullptr && N != 1)) return METEORA_ERR_INVALID_ARG;
    const meteora_status s = check_i8_weights(W, w_scale, T, d_in, d_out, dt, out);
    if (s != METEORA_OK) return s;
    if (N > kMaxAdapters || !aligned(q, 16) || !aligned(q_scale, 16) || (offsets && !aligned(offsets, 4)))
        return METEORA_ERR_UNSUPPORTED;
    if (T == 0) return METEORA_OK;
    return status(launch_gemm_i8(q, q_scale, W, w_scale, offsets, T, d_in, d_out, N, dt == METEORA_BF16, out,
                                 static_cast<hipStream_t>(stream)));
}

int meteora_gemm_i8_kernel(int T, int d_in, int d_out, int N, int grouped, const char** name, int* tile_rows, int* tile_cols,
                           int* per_cu, int* read_once, int* tail) {
    if (T < 1 || d_in < 1 || d_out < 1 || N < 1 || N > kMaxAdapters || (!grouped && N != 1) || !i8_sizes_supported(T, d_in, d_out))
        return -1;
    const I8Plan p = gemm_i8_plan(T, d_in, d_out, N, grouped != 0);
    if (name) *name = p.kernel;
    if (tile_rows) *tile_rows = p.rows;
    if (tile_cols) *tile_cols = p.cols;
    if (per_cu) *per_cu = p.per_cu;
    if (read_once) *read_once = p.once;
    if (tail) *tail = p.tail;
    return 0;
}

size_t meteora_base_gemm_i8_workspace_bytes(int T, int d_in) {
    if (T < 0 || T > kRowsMax || d_in < 1 || d_in % 16 != 0 || d_in > kI8MaxInputs) return 0;
    return base_gemm_i8_bytes(T, d_in) + 256;
}

meteora_status meteora_base_gemm_i8(const void* x, const int8_t* W, const float* w_scale, int T, int d_in, int d_out,
                                    meteora_dtype dt, void* out, void* ws, size_t ws_bytes, meteora_stream stream) {
    if (!x) return METEORA_ERR_INVALID_ARG;
    const meteora_status s = check_i8_weights(W, w_scale, T, d_in, d_out, dt, out);
    if (s != METEORA_OK) return s;
    if (!aligned(x, 16)) return METEORA_ERR_UNSUPPORTED;
    if (!ws || !aligned(ws, 256) || ws_bytes < base_gemm_i8_bytes(T, d_in)) return METEORA_ERR_WORKSPACE;
    if (T == 0) return METEORA_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (base_gemm_i8_in_one(T, d_in))
        return status(launch_base_gemm_i8_in_one(x, W, w_scale, T, d_in, d_out, dt == METEORA_BF16, out, st));
    int8_t* q = static_cast<int8_t*>(ws);
    float* scale = reinterpret_cast<float*>(q + align_up((size_t)T * d_in, 256));
    const hipError_t e = launch_quantize_rows(x, T, d_in, dt == METEORA_BF16, q, scale, st);
    if (e != hipSuccess) return METEORA_ERR_HIP;
    return status(launch_gemm_i8(q, scale, W, w_scale, nullptr, T, d_in, d_out, 1, dt == METEORA_BF16, out, st));
}

size_t meteora_sort_workspace_bytes(int T, int k, int N) {
    if (!sort_shape_ok(T, k, N) || !sort_shape_supported(T, k, N)) return 0;
    return align_up(sort_count_bytes(N), 256) + 256;
}

meteora_status meteora_sort_tokens(const void* x, const int32_t* topk_idx, int T, int k, int N, int d, meteora_dtype dt, void* xs,
                                   float* xs_scale, int32_t* pos, int32_t* offsets, void* ws, size_t ws_bytes,
                                   meteora_stream stream) {
    if (!x || !topk_idx || !xs || !pos || !offsets || !sort_shape_ok(T, k, N) || d < 1) return METEORA_ERR_INVALID_ARG;
    if (!known(dt) || !sort_shape_supported(T, k, N) || d % 8 != 0) return METEORA_ERR_UNSUPPORTED;
    if (!aligned(x, 16) || !aligned(topk_idx, 16) || !aligned(xs, 16) || !aligned(pos, 4) || !aligned(offsets, 4) ||
        (xs_scale && !aligned(xs_scale, 4)))
        return METEORA_ERR_UNSUPPORTED;
    if (!ws || !aligned(ws, 256) || (T > 0 && ws_bytes < sort_count_bytes(N))) return METEORA_ERR_WORKSPACE;
    if (T == 0) return METEORA_OK;
    return status(launch_sort_tokens(x, topk_idx, T, k, N, d, dt == METEORA_BF16, xs, xs_scale, pos, offsets,
                                     static_cast<int32_t*>(ws), static_cast<hipStream_t>(stream)));
}

static meteora_status check_unsort(const void* ys, int64_t rows, const int32_t* pos, const float* w, int T, int k, int d,
                                   float scale, meteora_dtype dt) {
    if ((!ys && rows > 0) || !pos || rows < 0 || T < 0 || k < 1 || d < 1 || !isfinite(scale)) return METEORA_ERR_INVALID_ARG;
    if (!known(dt) || k > kMaxTopK || T > kRowsMax || rows > INT32_MAX || d % 8 != 0)
        return METEORA_ERR_UNSUPPORTED;
    if (!aligned(ys, 16) || !aligned(pos, 4) || (w && !aligned(w, 4))) return METEORA_ERR_UNSUPPORTED;
    return METEORA_OK;
}

meteora_status meteora_unsort_tokens(const void* ys, int64_t rows, const int32_t* pos, const float* w, int T, int k, int d,
                                     float scale, meteora_dtype dt, const void* base, void* out, meteora_stream stream) {
    if (!out) return METEORA_ERR_INVALID_ARG;
    const meteora_status s = check_unsort(ys, rows, pos, w, T, k, d, scale, dt);
    if (s != METEORA_OK) return s;
    if (!aligned(out, 16) || (base && !aligned(base, 16))) return METEORA_ERR_UNSUPPORTED;
    if (T == 0) return METEORA_OK;
    return status(launch_unsort_tokens(ys, rows, pos, w, T, k, d, dt == METEORA_BF16, scale, base, out,
                                       static_cast<hipStream_t>(stream)));
}

meteora_status meteora_unsort_backward(const void* dy, const void* ys, int64_t rows, const int32_t* pos, const float* w, int T,
                                       int k, int d, float scale, meteora_dtype dt, void* dys, float* dw,
                                       meteora_stream stream) {
    if (!dy || (!dys && rows > 0)) return METEORA_ERR_INVALID_ARG;
    const meteora_status s = check_unsort(ys ? ys : (dw ? nullptr : dys), rows, pos, w, T, k, d, scale, dt);
    if (s != METEORA_OK) return s;
    if (!aligned(dy, 16) || !aligned(dys, 16) || (dw && !aligned(dw, 4))) return METEORA_ERR_UNSUPPORTED;
    if (T == 0) return METEORA_OK;
    return status(launch_unsort_backward(dy, ys, rows, pos, w, T, k, d, dt == METEORA_BF16, scale, dys, dw,
                                         static_cast<hipStream_t>(stream)));
}

}  // extern "C"
