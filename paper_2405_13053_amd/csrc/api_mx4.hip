// Entry points of the 4-bit rows and products (declared in include/meteora.h): argument validation and the launch sequence of each.  No
// device memory is allocated here and nothing synchronises with the host.
#include "../../include/meteora.h"
#include "common.hpp"
#include "kernels.hpp"
#include "quant_mx4.hpp"

using namespace meteora;

namespace {

constexpr int kMxMaxInputs = 131072, kMxMaxOutputs = 1 << 20;
constexpr int kRowsMax = (1 << 24) - 1;

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool known(meteora_dtype dt) { return dt == METEORA_F32 || dt == METEORA_BF16; }
inline meteora_status status(hipError_t e) { return e == hipSuccess ? METEORA_OK : METEORA_ERR_HIP; }

bool rows_supported(int rows, int d) {
    return d % kMxBlock == 0 && d <= kMxMaxInputs && rows <= kRowsMax && (int64_t)rows * d < (int64_t)1 << 36;
}
bool product_supported(int T, int d_in, int d_out) {
    return rows_supported(T, d_in) && d_out % 8 == 0 && d_out <= kMxMaxOutputs && (int64_t)T * d_out < (int64_t)1 << 33;
}
meteora_status check_weights(const uint8_t* W, const uint8_t* w_scale, int T, int d_in, int d_out, meteora_dtype dt, const void* out) {
    if (!W || !w_scale || !out || T < 0 || d_in < 1 || d_out < 1) return METEORA_ERR_INVALID_ARG;
    if (!known(dt) || !product_supported(T, d_in, d_out)) return METEORA_ERR_UNSUPPORTED;
    if (!aligned(W, 16) || !aligned(w_scale, 16) || !aligned(out, 16)) return METEORA_ERR_UNSUPPORTED;
    return METEORA_OK;
}
size_t base_gemm_bytes(int T, int d_in) {   // the quantised rows, then their scales
    return align_up((size_t)T * (d_in / 2), 256) + align_up(mx4_scale_bytes(T, d_in), 256);
}
// The gradient's: the transposed values, then (bf16) the parts of a split contraction, which numbers the outputs d_in.  Where it reads the codes
// themselves the parts are in the values' place; fp32 with more than few outputs reads nothing else, and has room for parts as large as up to 16384 outputs ask for
// (25.6 MB, at 100000 tokens of 32 inputs; a batch whose parts do not fit gets fewer of them).
constexpr size_t kBackParts = (size_t)32 << 20;
size_t values_bytes(int d_in, int d_out, meteora_dtype dt) {
    const size_t all = align_up((size_t)d_in * d_out * (dt == METEORA_BF16 ? 2 : 4), 256);
    return dt == METEORA_F32 && d_out > kMxBackFewOutputs && all > kBackParts ? kBackParts : all;
}
size_t splits_bytes(int T, int d_in, int d_out, meteora_dtype dt) {
    return dt == METEORA_BF16 && !mx4_back_takes(T, d_in, d_out, true) ? (size_t)gemm_few_tile_splits(T, d_out, d_in) * T * d_in * sizeof(float) : 0;
}

}  // namespace

extern "C" {

size_t meteora_mx4_scale_bytes(int rows, int d) {
    return rows < 0 || d < 1 || !rows_supported(rows, d) ? 0 : mx4_scale_bytes(rows, d);
}

meteora_status meteora_quantize_mx4(const void* x, int rows, int d, meteora_dtype dt, uint8_t* q, uint8_t* scale, meteora_stream stream) {
    if (!x || !q || !scale || rows < 0 || d < 1) return METEORA_ERR_INVALID_ARG;
    if (!known(dt) || !rows_supported(rows, d) || !aligned(x, 16) || !aligned(q, 16) || !aligned(scale, 16)) return METEORA_ERR_UNSUPPORTED;
    if (rows == 0) return METEORA_OK;
    return status(launch_quantize_mx4(x, rows, d, dt == METEORA_BF16, q, scale, static_cast<hipStream_t>(stream)));
}

meteora_status meteora_dequantize_mx4(const uint8_t* q, const uint8_t* scale, int rows, int d, meteora_dtype dt, int transpose, void* out,
                                      meteora_stream stream) {
    if (!q || !scale || !out || rows < 0 || d < 1) return METEORA_ERR_INVALID_ARG;
    if (!known(dt) || !rows_supported(rows, d) || (transpose && rows % 8 != 0) || !aligned(q, 16) || !aligned(scale, 16) || !aligned(out, 16))
        return METEORA_ERR_UNSUPPORTED;
    if (rows == 0) return METEORA_OK;
    return status(launch_dequantize_mx4(q, scale, rows, d, transpose != 0, dt == METEORA_BF16, out, static_cast<hipStream_t>(stream)));
}

meteora_status meteora_gemm_mx4(const uint8_t* q, const uint8_t* q_scale, const uint8_t* W, const uint8_t* w_scale, const int32_t* offsets,
                                int T, int d_in, int d_out, int N, meteora_dtype dt, void* out, meteora_stream stream) {
    if (!q || !q_scale || N < 1 || (offsets == nullptr && N != 1)) return METEORA_ERR_INVALID_ARG;
    const meteora_status s = check_weights(W, w_scale, T, d_in, d_out, dt, out);
    if (s != METEORA_OK) return s;
    if (N > kMaxAdapters || !aligned(q, 16) || !aligned(q_scale, 16) || (offsets && !aligned(offsets, 4))) return METEORA_ERR_UNSUPPORTED;
    if (T == 0) return METEORA_OK;
    return status(launch_gemm_mx4(q, q_scale, W, w_scale, offsets, T, d_in, d_out, N, dt == METEORA_BF16, out,
                                  static_cast<hipStream_t>(stream)));
}

int meteora_gemm_mx4_kernel(int T, int d_in, int d_out, int N, int grouped, const char** name, int* tile_rows, int* tile_cols, int* per_cu,
                            int* read_once, int* tail) {
    if (T < 1 || d_in < 1 || d_out < 1 || N < 1 || N > kMaxAdapters || (!grouped && N != 1) || !product_supported(T, d_in, d_out)) return -1;
    const I8Plan p = gemm_mx4_plan(T, d_in, d_out, N, grouped != 0);
    if (name) *name = p.kernel;
    if (tile_rows) *tile_rows = p.rows;
    if (tile_cols) *tile_cols = p.cols;
    if (per_cu) *per_cu = p.per_cu;
    if (read_once) *read_once = p.once;
    if (tail) *tail = p.tail;
    return 0;
}

size_t meteora_base_gemm_mx4_workspace_bytes(int T, int d_in) {
    return T < 0 || d_in < 1 || !rows_supported(T, d_in) ? 0 : base_gemm_bytes(T, d_in) + 256;
}

meteora_status meteora_base_gemm_mx4(const void* x, const uint8_t* W, const uint8_t* w_scale, int T, int d_in, int d_out, meteora_dtype dt,
                                     void* out, void* ws, size_t ws_bytes, meteora_stream stream) {
    if (!x) return METEORA_ERR_INVALID_ARG;
    const meteora_status s = check_weights(W, w_scale, T, d_in, d_out, dt, out);
    if (s != METEORA_OK) return s;
    if (!aligned(x, 16)) return METEORA_ERR_UNSUPPORTED;
    if (!ws || !aligned(ws, 256) || ws_bytes < base_gemm_bytes(T, d_in)) return METEORA_ERR_WORKSPACE;
    if (T == 0) return METEORA_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (base_gemm_mx4_in_one(T, d_in, d_out))
        return status(launch_base_gemm_mx4_in_one(x, W, w_scale, T, d_in, d_out, dt == METEORA_BF16, out, st));
    uint8_t* q = static_cast<uint8_t*>(ws);
    uint8_t* scale = q + align_up((size_t)T * (d_in / 2), 256);
    const hipError_t e = launch_quantize_mx4(x, T, d_in, dt == METEORA_BF16, q, scale, st);
    if (e != hipSuccess) return METEORA_ERR_HIP;
    return status(launch_gemm_mx4(q, scale, W, w_scale, nullptr, T, d_in, d_out, 1, dt == METEORA_BF16, out, st));
}

size_t meteora_base_gemm_mx4_backward_workspace_bytes(int d_in, int d_out, meteora_dtype dt) {
    if (d_in < 1 || d_out < 1 || !known(dt) || !product_supported(0, d_in, d_out)) return 0;
    return values_bytes(d_in, d_out, dt) + align_up(dt == METEORA_BF16 ? gemm_few_tile_bytes(kRowsMax, d_out, d_in) : 0, 256) + 256;
}

meteora_status meteora_base_gemm_mx4_backward(const void* dy, const uint8_t* W, const uint8_t* w_scale, int T, int d_in, int d_out,
                                              meteora_dtype dt, void* dx, void* ws, size_t ws_bytes, meteora_stream stream) {
    if (!dy) return METEORA_ERR_INVALID_ARG;
    const meteora_status s = check_weights(W, w_scale, T, d_in, d_out, dt, dx);
    if (s != METEORA_OK) return s;
    if (!aligned(dy, 16)) return METEORA_ERR_UNSUPPORTED;
    if (!ws || !aligned(ws, 256) || ws_bytes < values_bytes(d_in, d_out, dt) + splits_bytes(T, d_in, d_out, dt)) return METEORA_ERR_WORKSPACE;
    if (T == 0) return METEORA_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool bf16 = dt == METEORA_BF16;
    if (mx4_back_takes(T, d_in, d_out, bf16))
        return status(launch_mx4_back(dy, W, w_scale, T, d_in, d_out, bf16, dx, ws, values_bytes(d_in, d_out, dt), st));
    hipError_t e = launch_dequantize_mx4(W, w_scale, d_out, d_in, true, bf16, ws, st);
    if (e != hipSuccess) return METEORA_ERR_HIP;
    float* const splits = reinterpret_cast<float*>(static_cast<char*>(ws) + values_bytes(d_in, d_out, dt));
    if (bf16 && gemm_few_tile_splits(T, d_out, d_in) > 0)
        e = launch_gemm_few_tiles(dy, ws, T, d_out, d_in, nullptr, 0, nullptr, 0, dx, splits, st);
    else
        e = launch_gemm(dy, ws, T, d_out, d_in, bf16, nullptr, 0, nullptr, 0, dx, 0, nullptr, st);
    return status(e);
}

}  // extern "C"
