// C ABI of the calls that carry a gradient through a decoder layer: argument validation, workspace carving, sequencing.
#include <cmath>
#include <new>

#include "qless_kernels.h"
#include "tc_common.cuh"

namespace qless {

static bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

static qless_status check_workspace(const void* workspace, size_t given, size_t needed)
{
    if (needed == 0) return QLESS_OK;
    QLESS_REQUIRE(workspace != nullptr && aligned(workspace, 256), QLESS_ERR_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
    QLESS_REQUIRE(given >= needed, QLESS_ERR_WORKSPACE, "workspace too small: %zu bytes given, %zu needed", given, needed);
    return QLESS_OK;
}

// A bf16 matrix that is read or written in vectors and by tensor maps.
static qless_status check_matrix(const char* name, const void* p, int64_t ld, int64_t cols)
{
    QLESS_REQUIRE(p != nullptr, QLESS_ERR_INVALID_ARG, "%s is required", name);
    QLESS_REQUIRE(aligned(p, 16), QLESS_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
    QLESS_REQUIRE(ld >= cols && ld % 8 == 0 && ld < ((int64_t)1 << 38), QLESS_ERR_INVALID_ARG, "the row stride of %s must be at least %lld and a multiple of 8 (%lld)", name,
                  (long long)cols, (long long)ld);
    return QLESS_OK;
}

static qless_status check_norm(qless_dtype dtype, qless_dtype param_dtype, int64_t tokens, int32_t width)
{
    QLESS_REQUIRE(tokens >= 0 && width >= 1, QLESS_ERR_INVALID_ARG, "tokens must be >= 0 and width >= 1 (tokens=%lld, width=%d)", (long long)tokens, width);
    QLESS_REQUIRE((dtype == QLESS_F32 || dtype == QLESS_BF16) && (param_dtype == QLESS_F32 || param_dtype == QLESS_BF16), QLESS_ERR_INVALID_ARG,
                  "dtype and param_dtype must be QLESS_F32 or QLESS_BF16");
    QLESS_REQUIRE(width <= 16384, QLESS_ERR_UNSUPPORTED, "width must be at most 16384 (width=%d)", width);
    QLESS_REQUIRE(tokens < ((int64_t)1 << 31), QLESS_ERR_UNSUPPORTED, "tokens must be below 2^31");
    return QLESS_OK;
}

static qless_status check_heads(int64_t tokens, int64_t n, int32_t heads, int32_t kv_heads, int32_t head_dim)
{
    QLESS_REQUIRE(tokens >= 0 && n >= 0 && heads > 0 && kv_heads > 0 && head_dim > 0, QLESS_ERR_INVALID_ARG,
                  "tokens and n must be >= 0, heads, kv_heads and head_dim > 0 (tokens=%lld, n=%lld, heads=%d, kv_heads=%d, head_dim=%d)", (long long)tokens, (long long)n,
                  heads, kv_heads, head_dim);
    QLESS_REQUIRE(tokens < ((int64_t)1 << 31) && n < ((int64_t)1 << 31), QLESS_ERR_UNSUPPORTED, "tokens and n must be below 2^31");
    QLESS_REQUIRE(heads % kv_heads == 0 && heads <= 4096, QLESS_ERR_UNSUPPORTED, "heads must be a multiple of kv_heads, at most 4096 (heads=%d, kv_heads=%d)", heads, kv_heads);
    QLESS_REQUIRE(head_dim % 8 == 0 && head_dim <= 128, QLESS_ERR_UNSUPPORTED, "head_dim must be a multiple of 8, at most 128 (head_dim=%d)", head_dim);
    return QLESS_OK;
}

// An item of the kernels walks over an example's rows (a tile of keys: over those of every head of the group), and others of its block wait that long for
// the place it holds: at about 2 us for 128 rows, 2^25 rows take a quarter of the two seconds after which a wait gives up.
constexpr int64_t MOST_ROWS = (int64_t)1 << 25;

static qless_status check_offsets(const int64_t* offsets, int64_t tokens, int64_t n, int32_t group)
{
    QLESS_REQUIRE(offsets != nullptr, QLESS_ERR_INVALID_ARG, "offsets are required");
    QLESS_REQUIRE(offsets[0] >= 0 && offsets[n] <= tokens, QLESS_ERR_INVALID_ARG, "offsets must lie in [0, tokens]");
    for (int64_t e = 0; e < n; ++e)
        QLESS_REQUIRE(offsets[e] <= offsets[e + 1], QLESS_ERR_INVALID_ARG, "offsets must not decrease (offsets[%lld] > offsets[%lld])", (long long)e, (long long)e + 1);
    for (int64_t e = 0; e < n; ++e)
        QLESS_REQUIRE(offsets[e + 1] - offsets[e] <= MOST_ROWS / group, QLESS_ERR_UNSUPPORTED,
                      "an example's tokens times heads / kv_heads must be at most 2^25 (example %lld: %lld tokens)", (long long)e, (long long)(offsets[e + 1] - offsets[e]));
    return QLESS_OK;
}

static qless_status check_ffn(int64_t tokens, int32_t width, int32_t inner, qless_activation act)
{
    QLESS_REQUIRE(tokens >= 0 && width > 0 && inner > 0, QLESS_ERR_INVALID_ARG, "tokens must be >= 0, width and inner > 0 (tokens=%lld, width=%d, inner=%d)",
                  (long long)tokens, width, inner);
    QLESS_REQUIRE(act == QLESS_SILU || act == QLESS_GELU, QLESS_ERR_INVALID_ARG, "act must be QLESS_SILU or QLESS_GELU");
    QLESS_REQUIRE(tokens < ((int64_t)1 << 31) - 256, QLESS_ERR_UNSUPPORTED, "tokens must be below 2^31 - 256");
    QLESS_REQUIRE(width % 8 == 0 && inner % 8 == 0 && width <= (1 << 20) && inner <= (1 << 20), QLESS_ERR_UNSUPPORTED,
                  "width and inner must be multiples of 8, at most 2^20 (width=%d, inner=%d)", width, inner);
    return QLESS_OK;
}

#define QLESS_STEP(expr)                         \
    do {                                         \
        const qless_status s__ = (expr);         \
        if (s__ != QLESS_OK) return s__;         \
    } while (0)

}  // namespace qless

using namespace qless;

extern "C" {

// ---- layer normalisation -------------------------------------------------------------------------

size_t qless_layer_norm_backward_workspace(int64_t tokens, int32_t width, int32_t want_params)
{
    if (check_norm(QLESS_F32, QLESS_F32, tokens, width) != QLESS_OK || tokens == 0 || want_params == 0) return 0;
    return norm_most_workspace(tokens, width, want_params != 0);
}

qless_status qless_layer_norm(const void* x, qless_dtype dtype, int64_t tokens, int32_t width, int64_t ld_x, const void* weight, const void* bias,
                              qless_dtype param_dtype, float eps, int32_t center, void* out, int64_t ld_out, float* mean, float* rstd, void* cuda_stream)
{
    QLESS_STEP(check_norm(dtype, param_dtype, tokens, width));
    QLESS_REQUIRE(eps >= 0.0f && std::isfinite(eps), QLESS_ERR_INVALID_ARG, "eps must be finite and >= 0");
    if (tokens == 0) return QLESS_OK;
    const size_t es = dtype == QLESS_F32 ? 4 : 2, ps = param_dtype == QLESS_F32 ? 4 : 2;
    QLESS_REQUIRE(x && weight && out, QLESS_ERR_INVALID_ARG, "x, weight and out are required");
    QLESS_REQUIRE(ld_x >= width && ld_out >= width, QLESS_ERR_INVALID_ARG, "row strides must cover a row (ld_x=%lld, ld_out=%lld)", (long long)ld_x, (long long)ld_out);
    QLESS_REQUIRE(aligned(x, es) && aligned(out, es) && aligned(weight, ps) && aligned(bias, ps) && aligned(mean, 4) && aligned(rstd, 4), QLESS_ERR_INVALID_ARG,
                  "tensors must be aligned to their element type");
    NormArgs a{};
    a.x = x; a.weight = weight; a.bias = bias; a.out = out; a.mean = mean; a.rstd = rstd; a.tokens = tokens; a.ld_x = ld_x; a.ld_out = ld_out;
    a.width = width; a.center = center != 0; a.dtype = dtype; a.param_dtype = param_dtype; a.eps = eps;
    return launch_norm_forward(a, reinterpret_cast<cudaStream_t>(cuda_stream));
}

qless_status qless_layer_norm_backward(const void* grad_out, int64_t ld_grad_out, const void* x, qless_dtype dtype, int64_t tokens, int32_t width,
                                       int64_t ld_x, const void* weight, qless_dtype param_dtype, int32_t center, const float* mean, const float* rstd,
                                       void* grad_x, int64_t ld_grad_x, void* grad_weight, void* grad_bias, void* workspace, size_t workspace_bytes,
                                       void* cuda_stream)
{
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    QLESS_STEP(check_norm(dtype, param_dtype, tokens, width));
    const size_t es = dtype == QLESS_F32 ? 4 : 2, ps = param_dtype == QLESS_F32 ? 4 : 2;
    const bool params = grad_weight != nullptr || grad_bias != nullptr;
    QLESS_REQUIRE(aligned(grad_weight, ps) && aligned(grad_bias, ps), QLESS_ERR_INVALID_ARG, "tensors must be aligned to their element type");
    if (tokens == 0) {                    // the gradients of an empty sum
        if (grad_weight != nullptr) QLESS_CUDA_TRY(cudaMemsetAsync(grad_weight, 0, ps * (size_t)width, st));
        if (grad_bias != nullptr) QLESS_CUDA_TRY(cudaMemsetAsync(grad_bias, 0, ps * (size_t)width, st));
        return QLESS_OK;
    }
    QLESS_REQUIRE(grad_out && x && weight && rstd && grad_x && (mean || !center), QLESS_ERR_INVALID_ARG, "grad_out, x, weight, rstd, grad_x, and with center mean, are required");
    QLESS_REQUIRE(ld_x >= width && ld_grad_out >= width && ld_grad_x >= width, QLESS_ERR_INVALID_ARG,
                  "row strides must cover a row (ld_x=%lld, ld_grad_out=%lld, ld_grad_x=%lld)", (long long)ld_x, (long long)ld_grad_out, (long long)ld_grad_x);
    QLESS_REQUIRE(aligned(x, es) && aligned(grad_out, es) && aligned(grad_x, es) && aligned(weight, ps) && aligned(mean, 4) && aligned(rstd, 4), QLESS_ERR_INVALID_ARG,
                  "tensors must be aligned to their element type");
    NormArgs a{};
    a.x = x; a.dy = grad_out; a.weight = weight; a.out = grad_x; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
    a.grad_weight = grad_weight; a.grad_bias = grad_bias; a.tokens = tokens; a.ld_x = ld_x; a.ld_dy = ld_grad_out; a.ld_out = ld_grad_x;
    a.width = width; a.center = center != 0; a.dtype = dtype; a.param_dtype = param_dtype;
    if (params) QLESS_STEP(check_workspace(workspace, workspace_bytes, norm_workspace(a)));
    unsigned int* flag = timeout_flag_ptr();
    QLESS_REQUIRE(flag != nullptr, QLESS_ERR_CUDA, "cannot resolve the device timeout flag");
    return launch_norm_backward(a, reinterpret_cast<uint8_t*>(workspace), flag, st);
}

// ---- attention -----------------------------------------------------------------------------------

size_t qless_attention_workspace(int64_t tokens, int64_t n, int32_t heads, int32_t kv_heads)
{
    if (check_heads(tokens, n, heads, kv_heads, 8) != QLESS_OK) return 0;
    return attention_workspace(tokens, n, heads, kv_heads, false);
}

size_t qless_attention_backward_workspace(int64_t tokens, int64_t n, int32_t heads, int32_t kv_heads)
{
    if (check_heads(tokens, n, heads, kv_heads, 8) != QLESS_OK) return 0;
    return attention_workspace(tokens, n, heads, kv_heads, true);
}

qless_status qless_attention(const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v, const int64_t* offsets,
                             int64_t tokens, int64_t n, int32_t heads, int32_t kv_heads, int32_t head_dim, float scale, void* out, int64_t ld_out,
                             float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    QLESS_STEP(check_heads(tokens, n, heads, kv_heads, head_dim));
    QLESS_REQUIRE(std::isfinite(scale) && scale > 0.0f, QLESS_ERR_INVALID_ARG, "scale must be finite and positive");
    if (n == 0) return QLESS_OK;
    QLESS_STEP(check_offsets(offsets, tokens, n, heads / kv_heads));
    if (tokens == 0) return QLESS_OK;
    QLESS_STEP(check_matrix("q", q, ld_q, (int64_t)heads * head_dim));
    QLESS_STEP(check_matrix("k", k, ld_k, (int64_t)kv_heads * head_dim));
    QLESS_STEP(check_matrix("v", v, ld_v, (int64_t)kv_heads * head_dim));
    QLESS_STEP(check_matrix("out", out, ld_out, (int64_t)heads * head_dim));
    QLESS_REQUIRE(aligned(lse, 4), QLESS_ERR_INVALID_ARG, "lse must be 4-byte aligned");
    QLESS_STEP(check_workspace(workspace, workspace_bytes, attention_workspace(tokens, n, heads, kv_heads, false)));
    unsigned int* flag = timeout_flag_ptr();
    QLESS_REQUIRE(flag != nullptr, QLESS_ERR_CUDA, "cannot resolve the device timeout flag");
    AttnArgs a{};
    a.q = q; a.k = k; a.v = v; a.ld_q = ld_q; a.ld_k = ld_k; a.ld_v = ld_v; a.out = out; a.ld_out = ld_out; a.lse = lse; a.offsets = offsets;
    a.tokens = tokens; a.n = n; a.heads = heads; a.kv_heads = kv_heads; a.head_dim = head_dim; a.scale = scale;
    try {
        return launch_attention(a, reinterpret_cast<uint8_t*>(workspace), flag, reinterpret_cast<cudaStream_t>(cuda_stream));
    } catch (const std::bad_alloc&) {
        return fail(QLESS_ERR_INVALID_ARG, "out of host memory for the tables of %lld examples", (long long)n);
    }
}

qless_status qless_attention_backward(const void* grad_out, int64_t ld_grad_out, const void* q, int64_t ld_q, const void* k, int64_t ld_k,
                                      const void* v, int64_t ld_v, const void* out, int64_t ld_out, const float* lse, const int64_t* offsets,
                                      int64_t tokens, int64_t n, int32_t heads, int32_t kv_heads, int32_t head_dim, float scale, void* grad_q,
                                      int64_t ld_grad_q, void* grad_k, int64_t ld_grad_k, void* grad_v, int64_t ld_grad_v, void* workspace,
                                      size_t workspace_bytes, void* cuda_stream)
{
    QLESS_STEP(check_heads(tokens, n, heads, kv_heads, head_dim));
    QLESS_REQUIRE(std::isfinite(scale) && scale > 0.0f, QLESS_ERR_INVALID_ARG, "scale must be finite and positive");
    if (n == 0) return QLESS_OK;
    QLESS_STEP(check_offsets(offsets, tokens, n, heads / kv_heads));
    if (tokens == 0) return QLESS_OK;
    const int64_t wide = (int64_t)heads * head_dim, narrow = (int64_t)kv_heads * head_dim;
    QLESS_STEP(check_matrix("grad_out", grad_out, ld_grad_out, wide));
    QLESS_STEP(check_matrix("q", q, ld_q, wide));
    QLESS_STEP(check_matrix("k", k, ld_k, narrow));
    QLESS_STEP(check_matrix("v", v, ld_v, narrow));
    QLESS_STEP(check_matrix("out", out, ld_out, wide));
    QLESS_STEP(check_matrix("grad_q", grad_q, ld_grad_q, wide));
    QLESS_STEP(check_matrix("grad_k", grad_k, ld_grad_k, narrow));
    QLESS_STEP(check_matrix("grad_v", grad_v, ld_grad_v, narrow));
    QLESS_REQUIRE(lse != nullptr && aligned(lse, 4), QLESS_ERR_INVALID_ARG, "lse is required, 4-byte aligned");
    QLESS_STEP(check_workspace(workspace, workspace_bytes, attention_workspace(tokens, n, heads, kv_heads, true)));
    unsigned int* flag = timeout_flag_ptr();
    QLESS_REQUIRE(flag != nullptr, QLESS_ERR_CUDA, "cannot resolve the device timeout flag");
    AttnArgs a{};
    a.q = q; a.k = k; a.v = v; a.out_in = out; a.dout = grad_out; a.ld_q = ld_q; a.ld_k = ld_k; a.ld_v = ld_v; a.ld_out = ld_out; a.ld_dout = ld_grad_out;
    a.lse_in = lse; a.dq = grad_q; a.dk = grad_k; a.dv = grad_v; a.ld_dq = ld_grad_q; a.ld_dk = ld_grad_k; a.ld_dv = ld_grad_v; a.offsets = offsets;
    a.tokens = tokens; a.n = n; a.heads = heads; a.kv_heads = kv_heads; a.head_dim = head_dim; a.scale = scale;
    try {
        return launch_attention_backward(a, reinterpret_cast<uint8_t*>(workspace), flag, reinterpret_cast<cudaStream_t>(cuda_stream));
    } catch (const std::bad_alloc&) {
        return fail(QLESS_ERR_INVALID_ARG, "out of host memory for the tables of %lld examples", (long long)n);
    }
}

// ---- gated feed-forward block --------------------------------------------------------------------

size_t qless_gated_ffn_workspace(int64_t tokens, int32_t width, int32_t inner)
{
    if (check_ffn(tokens, width, inner, QLESS_SILU) != QLESS_OK) return 0;
    return ffn_workspace(tokens, width, inner, false, false);
}

size_t qless_gated_ffn_backward_workspace(int64_t tokens, int32_t width, int32_t inner, int32_t want_weights)
{
    if (check_ffn(tokens, width, inner, QLESS_SILU) != QLESS_OK) return 0;
    return ffn_workspace(tokens, width, inner, true, want_weights != 0);
}

qless_status qless_gated_ffn(const void* x, int64_t ld_x, const void* w_gate, int64_t ld_w_gate, const void* w_up, int64_t ld_w_up,
                             const void* w_down, int64_t ld_w_down, int64_t tokens, int32_t width, int32_t inner, qless_activation act, void* out,
                             int64_t ld_out, void* hidden, int64_t ld_hidden, void* gate, int64_t ld_gate, void* up, int64_t ld_up, void* workspace,
                             size_t workspace_bytes, void* cuda_stream)
{
    QLESS_STEP(check_ffn(tokens, width, inner, act));
    if (tokens == 0) return QLESS_OK;
    QLESS_STEP(check_matrix("x", x, ld_x, width));
    QLESS_STEP(check_matrix("w_gate", w_gate, ld_w_gate, width));
    QLESS_STEP(check_matrix("w_up", w_up, ld_w_up, width));
    QLESS_STEP(check_matrix("w_down", w_down, ld_w_down, inner));
    QLESS_STEP(check_matrix("out", out, ld_out, width));
    QLESS_STEP(check_matrix("hidden", hidden, ld_hidden, inner));
    QLESS_REQUIRE((gate == nullptr) == (up == nullptr), QLESS_ERR_INVALID_ARG, "gate and up are kept together or not at all");
    if (gate != nullptr) {
        QLESS_STEP(check_matrix("gate", gate, ld_gate, inner));
        QLESS_STEP(check_matrix("up", up, ld_up, inner));
    }
    QLESS_STEP(check_workspace(workspace, workspace_bytes, ffn_workspace(tokens, width, inner, false, false)));
    unsigned int* flag = timeout_flag_ptr();
    QLESS_REQUIRE(flag != nullptr, QLESS_ERR_CUDA, "cannot resolve the device timeout flag");
    FfnArgs a{};
    a.x = x; a.w_gate = w_gate; a.w_up = w_up; a.w_down = w_down; a.ld_x = ld_x; a.ld_wg = ld_w_gate; a.ld_wu = ld_w_up; a.ld_wd = ld_w_down;
    a.out = out; a.hidden = hidden; a.gate = gate; a.up = up; a.ld_out = ld_out; a.ld_hidden = ld_hidden; a.ld_gate = ld_gate; a.ld_up = ld_up;
    a.tokens = tokens; a.width = width; a.inner = inner; a.act = act;
    return launch_ffn_forward(a, reinterpret_cast<uint8_t*>(workspace), flag, reinterpret_cast<cudaStream_t>(cuda_stream));
}

qless_status qless_gated_ffn_backward(const void* grad_out, int64_t ld_grad_out, const void* x, int64_t ld_x, const void* gate, int64_t ld_gate,
                                      const void* up, int64_t ld_up, const void* w_gate, int64_t ld_w_gate, const void* w_up, int64_t ld_w_up,
                                      const void* w_down, int64_t ld_w_down, int64_t tokens, int32_t width, int32_t inner, qless_activation act,
                                      void* grad_x, int64_t ld_grad_x, void* grad_gate, int64_t ld_grad_gate, void* grad_up, int64_t ld_grad_up,
                                      void* grad_w_gate, int64_t ld_grad_w_gate, void* grad_w_up, int64_t ld_grad_w_up, void* grad_w_down,
                                      int64_t ld_grad_w_down, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    QLESS_STEP(check_ffn(tokens, width, inner, act));
    if (grad_w_gate != nullptr) QLESS_STEP(check_matrix("grad_w_gate", grad_w_gate, ld_grad_w_gate, width));
    if (grad_w_up != nullptr) QLESS_STEP(check_matrix("grad_w_up", grad_w_up, ld_grad_w_up, width));
    if (grad_w_down != nullptr) QLESS_STEP(check_matrix("grad_w_down", grad_w_down, ld_grad_w_down, inner));
    if (tokens == 0) {                    // the gradients of an empty sum
        if (grad_w_gate != nullptr) QLESS_CUDA_TRY(cudaMemset2DAsync(grad_w_gate, (size_t)ld_grad_w_gate * 2, 0, (size_t)width * 2, (size_t)inner, st));
        if (grad_w_up != nullptr) QLESS_CUDA_TRY(cudaMemset2DAsync(grad_w_up, (size_t)ld_grad_w_up * 2, 0, (size_t)width * 2, (size_t)inner, st));
        if (grad_w_down != nullptr) QLESS_CUDA_TRY(cudaMemset2DAsync(grad_w_down, (size_t)ld_grad_w_down * 2, 0, (size_t)inner * 2, (size_t)width, st));
        return QLESS_OK;
    }
    const bool weights = grad_w_gate != nullptr || grad_w_up != nullptr || grad_w_down != nullptr;
    // (a tile of a weight's gradient is one contraction over the tokens, and its epilogue waits for it: 2^20 stages, half a second)
    QLESS_REQUIRE(!weights || tokens <= ((int64_t)1 << 27), QLESS_ERR_UNSUPPORTED, "tokens must be at most 2^27 where weights' gradients are wanted");
    QLESS_STEP(check_matrix("grad_out", grad_out, ld_grad_out, width));
    if (grad_w_gate != nullptr || grad_w_up != nullptr) QLESS_STEP(check_matrix("x", x, ld_x, width));
    QLESS_STEP(check_matrix("gate", gate, ld_gate, inner));
    QLESS_STEP(check_matrix("up", up, ld_up, inner));
    QLESS_STEP(check_matrix("w_gate", w_gate, ld_w_gate, width));
    QLESS_STEP(check_matrix("w_up", w_up, ld_w_up, width));
    QLESS_STEP(check_matrix("w_down", w_down, ld_w_down, inner));
    QLESS_STEP(check_matrix("grad_gate", grad_gate, ld_grad_gate, inner));
    QLESS_STEP(check_matrix("grad_up", grad_up, ld_grad_up, inner));
    if (grad_x != nullptr) QLESS_STEP(check_matrix("grad_x", grad_x, ld_grad_x, width));
    QLESS_STEP(check_workspace(workspace, workspace_bytes, ffn_workspace(tokens, width, inner, true, weights)));
    unsigned int* flag = timeout_flag_ptr();
    QLESS_REQUIRE(flag != nullptr, QLESS_ERR_CUDA, "cannot resolve the device timeout flag");
    FfnArgs a{};
    a.dy = grad_out; a.x = x; a.gate_in = gate; a.up_in = up; a.w_gate = w_gate; a.w_up = w_up; a.w_down = w_down;
    a.ld_dy = ld_grad_out; a.ld_x = ld_x; a.ld_gate_in = ld_gate; a.ld_up_in = ld_up; a.ld_wg = ld_w_gate; a.ld_wu = ld_w_up; a.ld_wd = ld_w_down;
    a.out = grad_x; a.gate = grad_gate; a.up = grad_up; a.ld_out = ld_grad_x; a.ld_gate = ld_grad_gate; a.ld_up = ld_grad_up;
    a.dw_gate = grad_w_gate; a.dw_up = grad_w_up; a.dw_down = grad_w_down; a.ld_dwg = ld_grad_w_gate; a.ld_dwu = ld_grad_w_up; a.ld_dwd = ld_grad_w_down;
    a.tokens = tokens; a.width = width; a.inner = inner; a.act = act;
    return launch_ffn_backward(a, reinterpret_cast<uint8_t*>(workspace), flag, st);
}

}  // extern "C"
