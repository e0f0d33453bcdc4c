// Entry points of the mixture of experts for a few tokens (declared in include/meteora.h): argument validation and the launch sequence.
// No device memory is allocated here and nothing synchronises with the host.
#include <math.h>

#include "../../include/meteora.h"
#include "common.hpp"
#include "kernels.hpp"
#include "quant_mx4.hpp"

using namespace meteora;

namespace {

constexpr int kExpertsMaxWidth = 131072;

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline meteora_status status(hipError_t e) { return e == hipSuccess ? METEORA_OK : METEORA_ERR_HIP; }

bool sizes_ok(int T, int d, int f, int N, int k) { return T >= 0 && d >= 1 && f >= 1 && N >= 1 && k >= 1; }
bool sizes_supported(int T, int d, int f, int N, int k) {
    return T <= kExpertsMaxTokens && N <= kMaxAdapters && k <= kMaxTopK && d % 8 == 0 && f % 8 == 0 && d <= kExpertsMaxWidth &&
           f <= kExpertsMaxWidth;
}
struct Scratch { size_t h, y, plan, idx, w, part, total; };
Scratch carve(int T, int d, int f, int N, int k) {   // idx, w, part: the routing of meteora_moe_forward
    Scratch s{};
    s.y = align_up(experts_h_bytes(T, k, f), 256);
    s.plan = s.y + align_up(experts_y_bytes(T, k, d), 256);
    s.idx = s.plan + align_up(experts_plan_bytes(), 256);
    s.w = s.idx + align_up((size_t)T * k * sizeof(int32_t), 256);
    s.part = s.w + align_up((size_t)T * k * sizeof(float), 256);
    s.total = s.part + align_up(experts_part_bytes(T, d, N), 256);
    return s;
}
// Everything but the routing's pointers
meteora_status check(const void* x, const void* W1, const uint8_t* s1, const void* W2, const uint8_t* s2, int T, int d, int f, int N, int k,
                     float scale, meteora_dtype dt, const void* base, const void* out, const void* ws, size_t ws_bytes) {
    if (!x || !W1 || !W2 || !out || !sizes_ok(T, d, f, N, k) || !isfinite(scale) || (s1 == nullptr) != (s2 == nullptr))
        return METEORA_ERR_INVALID_ARG;
    if (dt != METEORA_BF16 || !sizes_supported(T, d, f, N, k) || (s1 && (d % kMxBlock != 0 || f % kMxBlock != 0)))
        return METEORA_ERR_UNSUPPORTED;
    for (const void* p : {x, W1, (const void*)s1, W2, (const void*)s2, base, out})
        if (!aligned(p, 16)) return METEORA_ERR_UNSUPPORTED;
    if (!ws || !aligned(ws, 256) || ws_bytes < carve(T, d, f, N, k).total) return METEORA_ERR_WORKSPACE;
    return METEORA_OK;
}
ExpertsArgs arguments(const void* x, int32_t* idx, float* w, const void* W1, const uint8_t* s1, const void* W2, const uint8_t* s2,
                      int T, int d, int f, int N, int k, float scale, const void* base, void* out, void* ws) {
    const Scratch s = carve(T, d, f, N, k);
    char* const p = static_cast<char*>(ws);
    return {static_cast<const bf16_t*>(x), idx, w, static_cast<const uint8_t*>(W1), s1, static_cast<const uint8_t*>(W2), s2,
            static_cast<const bf16_t*>(base), static_cast<bf16_t*>(out), reinterpret_cast<bf16_t*>(p), reinterpret_cast<float*>(p + s.y), p + s.plan, scale,
            T, k, N, d, f, nullptr, nullptr, nullptr, 1.f};
}

}  // namespace

extern "C" {

size_t meteora_experts_workspace_bytes(int T, int d, int f, int N, int k) {
    if (!sizes_ok(T, d, f, N, k) || !sizes_supported(T, d, f, N, k)) return 0;
    return carve(T, d, f, N, k).total + 256;
}

meteora_status meteora_experts_forward(const void* x, const int32_t* topk_idx, const float* topk_w, const void* W1, const uint8_t* w1_scale,
                                       const void* W2, const uint8_t* w2_scale, int T, int d, int f, int N, int k, float scale,
                                       meteora_dtype dt, const void* base, void* out, void* ws, size_t ws_bytes, meteora_stream stream) {
    if (!topk_idx || !topk_w) return METEORA_ERR_INVALID_ARG;
    const meteora_status s = check(x, W1, w1_scale, W2, w2_scale, T, d, f, N, k, scale, dt, base, out, ws, ws_bytes);
    if (s != METEORA_OK) return s;
    if (!aligned(topk_idx, 4) || !aligned(topk_w, 4)) return METEORA_ERR_UNSUPPORTED;
    if (T == 0) return METEORA_OK;
    return status(launch_experts(arguments(x, const_cast<int32_t*>(topk_idx), const_cast<float*>(topk_w), W1, w1_scale, W2, w2_scale, T, d, f, N, k, scale, base, out, ws),
                                 static_cast<hipStream_t>(stream)));
}

meteora_status meteora_moe_forward(const void* x, const float* W_gate, const float* gate_bias, const void* W1, const uint8_t* w1_scale,
                                   const void* W2, const uint8_t* w2_scale, int T, int d, int f, int N, int k, float scale,
                                   float inv_temperature, meteora_dtype dt, const void* base, void* out, int32_t* topk_idx_out,
                                   float* topk_w_out, void* ws, size_t ws_bytes, meteora_stream stream) {
    if (!W_gate || !isfinite(inv_temperature) || k > N) return METEORA_ERR_INVALID_ARG;
    const meteora_status s = check(x, W1, w1_scale, W2, w2_scale, T, d, f, N, k, scale, dt, base, out, ws, ws_bytes);
    if (s != METEORA_OK) return s;
    if (!aligned(W_gate, 16) || !aligned(gate_bias, 4) || !aligned(topk_idx_out, 4) || !aligned(topk_w_out, 4)) return METEORA_ERR_UNSUPPORTED;
    if (T == 0) return METEORA_OK;
    const Scratch c = carve(T, d, f, N, k);
    int32_t* idx = topk_idx_out ? topk_idx_out : reinterpret_cast<int32_t*>(static_cast<char*>(ws) + c.idx);
    float* w = topk_w_out ? topk_w_out : reinterpret_cast<float*>(static_cast<char*>(ws) + c.w);
    ExpertsArgs a = arguments(x, idx, w, W1, w1_scale, W2, w2_scale, T, d, f, N, k, scale, base, out, ws);
    a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + c.part);
    a.W_gate = W_gate;
    a.bias = gate_bias;
    a.inv_temperature = inv_temperature;
    return status(launch_experts(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
