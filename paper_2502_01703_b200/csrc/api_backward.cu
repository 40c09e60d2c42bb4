// C ABI of the calls that produce gradient rows: argument validation, workspace carving, sequencing.
#include <algorithm>
#include <new>
#include <vector>

#include "qless_kernels.h"
#include "tc_common.cuh"

namespace qless {

static bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

static qless_status check_activation(qless_dtype dtype, int64_t tokens, int32_t width, int64_t ld_x, int32_t group, int64_t ld_codes,
                                     int64_t ld_scales)
{
    QLESS_REQUIRE(tokens >= 0 && width >= 1, QLESS_ERR_INVALID_ARG, "tokens must be >= 0 and width >= 1 (tokens=%lld, width=%d)", (long long)tokens, width);
    QLESS_REQUIRE(dtype == QLESS_F32 || dtype == QLESS_BF16, QLESS_ERR_INVALID_ARG, "dtype must be QLESS_F32 or QLESS_BF16");
    QLESS_REQUIRE(group == 32 || group == 64 || group == 128, QLESS_ERR_UNSUPPORTED, "group must be 32, 64 or 128 (group=%d)", group);
    QLESS_REQUIRE(width <= (1 << 24), QLESS_ERR_UNSUPPORTED, "width must be at most 2^24 (width=%d)", width);
    QLESS_REQUIRE(ld_x >= width && ld_codes >= width && ld_scales >= (width + group - 1) / group, QLESS_ERR_INVALID_ARG,
                  "row strides must cover a row (ld_x=%lld, ld_codes=%lld, ld_scales=%lld)", (long long)ld_x, (long long)ld_codes, (long long)ld_scales);
    return QLESS_OK;
}

}  // namespace qless

using namespace qless;

extern "C" {

// ---- activation checkpoints --------------------------------------------------------------------

qless_status qless_activation_quantize(const void* x, qless_dtype dtype, int64_t tokens, int32_t width, int64_t ld_x, int32_t group,
                                       int8_t* codes, int64_t ld_codes, uint8_t* scales, int64_t ld_scales, void* cuda_stream)
{
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    qless_status s = check_activation(dtype, tokens, width, ld_x, group, ld_codes, ld_scales);
    if (s != QLESS_OK) return s;
    if (tokens == 0) return QLESS_OK;
    QLESS_REQUIRE(x != nullptr && codes != nullptr && scales != nullptr, QLESS_ERR_INVALID_ARG, "x, codes and scales are required");
    QLESS_REQUIRE(aligned(x, dtype == QLESS_F32 ? 4 : 2), QLESS_ERR_INVALID_ARG, "x must be aligned to its element type");
    ProfileScope ps("activation_quantize", st);
    QLESS_CUDA_TRY(launch_activation_quantize(x, dtype, tokens, width, ld_x, group, codes, ld_codes, scales, ld_scales, st));
    return QLESS_OK;
}

qless_status qless_activation_dequantize(const int8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t ld_scales, int64_t tokens,
                                         int32_t width, int32_t group, void* x, qless_dtype dtype, int64_t ld_x, void* cuda_stream)
{
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    qless_status s = check_activation(dtype, tokens, width, ld_x, group, ld_codes, ld_scales);
    if (s != QLESS_OK) return s;
    if (tokens == 0) return QLESS_OK;
    QLESS_REQUIRE(x != nullptr && codes != nullptr && scales != nullptr, QLESS_ERR_INVALID_ARG, "x, codes and scales are required");
    QLESS_REQUIRE(aligned(x, dtype == QLESS_F32 ? 4 : 2), QLESS_ERR_INVALID_ARG, "x must be aligned to its element type");
    ProfileScope ps("activation_dequantize", st);
    QLESS_CUDA_TRY(launch_activation_dequantize(codes, ld_codes, scales, ld_scales, tokens, width, group, x, dtype, ld_x, st));
    return QLESS_OK;
}

// ---- per-example LoRA gradients ------------------------------------------------------------------

static qless_status check_lora_shape(int64_t tokens, int64_t n, int32_t in, int32_t out, int32_t rank, qless_dtype dtype)
{
    QLESS_REQUIRE(tokens >= 0 && n >= 0 && in > 0 && out > 0 && rank > 0, QLESS_ERR_INVALID_ARG,
                  "tokens and n must be >= 0, in, out and rank > 0 (tokens=%lld, n=%lld, in=%d, out=%d, rank=%d)", (long long)tokens, (long long)n, in, out, rank);
    QLESS_REQUIRE(dtype == QLESS_F32 || dtype == QLESS_BF16, QLESS_ERR_INVALID_ARG, "dtype must be QLESS_F32 or QLESS_BF16");
    QLESS_REQUIRE(tokens < ((int64_t)1 << 31) && n < ((int64_t)1 << 31), QLESS_ERR_UNSUPPORTED, "tokens and n must be below 2^31");
    QLESS_REQUIRE(in % 16 == 0 && out % 16 == 0 && in <= (1 << 20) && out <= (1 << 20), QLESS_ERR_UNSUPPORTED,
                  "in and out must be multiples of 16, at most 2^20 (in=%d, out=%d)", in, out);
    QLESS_REQUIRE(rank % 8 == 0 && rank <= 128, QLESS_ERR_UNSUPPORTED, "rank must be a multiple of 8, at most 128 (rank=%d)", rank);
    return QLESS_OK;
}

size_t qless_lora_gradients_workspace(int64_t tokens, int64_t n, int32_t in, int32_t out, int32_t rank, qless_dtype dtype)
{
    if (check_lora_shape(tokens, n, in, out, rank, dtype) != QLESS_OK) return 256;
    return plan_lora(tokens, n, in, out, rank, dtype).total;
}

qless_status qless_lora_gradients(const int8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t ld_scales, int32_t group,
                                  const void* grad_out, int64_t ld_grad_out, const void* lora_a, const void* lora_b,
                                  const int64_t* offsets, int64_t tokens, int64_t n, int32_t in, int32_t out, int32_t rank, float scaling,
                                  void* grads, qless_dtype dtype, int64_t ld_grads, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    qless_status s = check_lora_shape(tokens, n, in, out, rank, dtype);
    if (s != QLESS_OK) return s;
    s = check_activation(QLESS_BF16, tokens, in, in, group, ld_codes, ld_scales);
    if (s != QLESS_OK) return s;
    if (n == 0) return QLESS_OK;
    QLESS_REQUIRE(offsets != nullptr && grads != nullptr, QLESS_ERR_INVALID_ARG, "offsets and grads are required");
    QLESS_REQUIRE(offsets[0] >= 0 && offsets[n] <= tokens, QLESS_ERR_INVALID_ARG, "offsets must lie in [0, tokens]");
    for (int64_t e = 0; e < n; ++e)
        QLESS_REQUIRE(offsets[e] <= offsets[e + 1], QLESS_ERR_INVALID_ARG, "offsets must not decrease (offsets[%lld] > offsets[%lld])", (long long)e, (long long)e + 1);
    if (tokens > 0) {
        QLESS_REQUIRE(codes && scales && grad_out && lora_a && lora_b, QLESS_ERR_INVALID_ARG, "codes, scales, grad_out, lora_a and lora_b are required");
        QLESS_REQUIRE(aligned(codes, 16) && aligned(grad_out, 16) && aligned(lora_a, 16) && aligned(lora_b, 16), QLESS_ERR_INVALID_ARG,
                      "codes, grad_out, lora_a and lora_b must be 16-byte aligned");
        QLESS_REQUIRE(ld_codes % 16 == 0 && ld_grad_out >= out && ld_grad_out % 8 == 0, QLESS_ERR_INVALID_ARG,
                      "ld_codes must be a multiple of 16, ld_grad_out >= out and a multiple of 8 (ld_codes=%lld, ld_grad_out=%lld)", (long long)ld_codes, (long long)ld_grad_out);
    }
    QLESS_REQUIRE(aligned(grads, 16) && ld_grads >= (int64_t)rank * (in + out) && ld_grads % 8 == 0, QLESS_ERR_INVALID_ARG,
                  "grads must be 16-byte aligned, ld_grads >= rank * (in + out) and a multiple of 8 (ld_grads=%lld)", (long long)ld_grads);
    const LoraPlan pl = plan_lora(tokens, n, in, out, rank, dtype);
    QLESS_REQUIRE(workspace != nullptr && aligned(workspace, 256), QLESS_ERR_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
    QLESS_REQUIRE(workspace_bytes >= pl.total, QLESS_ERR_WORKSPACE, "workspace too small: %zu bytes given, %zu needed", workspace_bytes, pl.total);
    unsigned int* flag = timeout_flag_ptr();
    QLESS_REQUIRE(flag != nullptr, QLESS_ERR_CUDA, "cannot resolve the device timeout flag");
    try {
        std::vector<LoraChunk> chunks;
        std::vector<LoraJoin> joins;
        chunks.reserve((size_t)n + 64);
        int32_t slots = 0;
        for (int64_t e = 0; e < n; ++e) {
            const int64_t len = offsets[e + 1] - offsets[e];
            if (len <= pl.chunk) {
                chunks.push_back({offsets[e], (int32_t)len, (int32_t)e, -1, 0});
                continue;
            }
            const int64_t pieces = (len + pl.chunk - 1) / pl.chunk;
            joins.push_back({(int32_t)e, slots, (int32_t)pieces, 0});
            for (int64_t k = 0; k < pieces; ++k) {
                const int64_t t0 = k * pl.chunk;
                chunks.push_back({offsets[e] + t0, (int32_t)(len - t0 < pl.chunk ? len - t0 : pl.chunk), (int32_t)e, slots++, 0});
            }
        }
        // Long pieces first: the blocks take the items in turn, and the last rounds are then short (385 instead of 397 us for 128 examples of
        // 130 to 900 tokens, 139 instead of 148 us for 32).
        std::stable_sort(chunks.begin(), chunks.end(), [](const LoraChunk& x, const LoraChunk& y) { return x.len > y.len; });
        LoraArgs a;
        a.codes = codes; a.scales = scales; a.grad_out = grad_out; a.lora_a = lora_a; a.lora_b = lora_b;
        a.T = tokens; a.ld_codes = ld_codes; a.ld_scales = ld_scales; a.ld_grad_out = ld_grad_out; a.ld_grads = ld_grads;
        a.in = in; a.out = out; a.rank = rank; a.group = group; a.scaling = scaling; a.dtype = dtype; a.grads = grads;
        a.chunks = chunks.data(); a.joins = joins.data();
        a.num_chunks = (int64_t)chunks.size(); a.num_joins = (int64_t)joins.size();
        return launch_lora(a, pl, reinterpret_cast<uint8_t*>(workspace), flag, st);
    } catch (const std::bad_alloc&) {
        return fail(QLESS_ERR_INVALID_ARG, "out of host memory for the tables of %lld examples", (long long)n);
    }
}

// ---- loss of the language model's head -----------------------------------------------------------

static qless_status check_loss_shape(int64_t tokens, int32_t width, int32_t vocab)
{
    QLESS_REQUIRE(tokens >= 0 && width > 0 && vocab > 0, QLESS_ERR_INVALID_ARG, "tokens must be >= 0, width and vocab > 0 (tokens=%lld, width=%d, vocab=%d)",
                  (long long)tokens, width, vocab);
    QLESS_REQUIRE(tokens < ((int64_t)1 << 31) - 256 && vocab < 0x7FFFFFFF - 256, QLESS_ERR_UNSUPPORTED, "tokens and vocab must be below 2^31 - 256");
    QLESS_REQUIRE(width % 8 == 0 && width <= 65536, QLESS_ERR_UNSUPPORTED, "width must be a multiple of 8, at most 65536 (width=%d)", width);
    return QLESS_OK;
}

size_t qless_lm_loss_workspace(int64_t tokens, int32_t width, int32_t vocab, int32_t want_hidden, int32_t want_weight)
{
    if (check_loss_shape(tokens, width, vocab) != QLESS_OK || tokens == 0) return 256;
    return plan_loss(tokens, width, vocab, want_hidden != 0, want_weight != 0).total;
}

qless_status qless_lm_loss(const void* hidden, int64_t ld_hidden, const void* weight, int64_t ld_weight, const int64_t* labels,
                           const float* token_weight, int64_t tokens, int32_t width, int32_t vocab, float* loss, void* grad_hidden,
                           int64_t ld_grad_hidden, void* grad_weight, int64_t ld_grad_weight, void* workspace, size_t workspace_bytes,
                           void* cuda_stream)
{
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    qless_status s = check_loss_shape(tokens, width, vocab);
    if (s != QLESS_OK) return s;
    QLESS_REQUIRE(grad_weight == nullptr || (aligned(grad_weight, 16) && ld_grad_weight >= width && ld_grad_weight % 8 == 0), QLESS_ERR_INVALID_ARG,
                  "grad_weight must be 16-byte aligned, ld_grad_weight >= width and a multiple of 8 (ld_grad_weight=%lld)", (long long)ld_grad_weight);
    if (tokens == 0) {                    // the gradient of an empty sum
        if (grad_weight != nullptr) QLESS_CUDA_TRY(cudaMemset2DAsync(grad_weight, (size_t)ld_grad_weight * 2, 0, (size_t)width * 2, (size_t)vocab, st));
        return QLESS_OK;
    }
    QLESS_REQUIRE(hidden && weight && labels && loss, QLESS_ERR_INVALID_ARG, "hidden, weight, labels and loss are required");
    QLESS_REQUIRE(aligned(hidden, 16) && aligned(weight, 16) && aligned(labels, 8), QLESS_ERR_INVALID_ARG,
                  "hidden and weight must be 16-byte aligned, labels 8-byte aligned");
    QLESS_REQUIRE(ld_hidden >= width && ld_hidden % 8 == 0 && ld_weight >= width && ld_weight % 8 == 0, QLESS_ERR_INVALID_ARG,
                  "ld_hidden and ld_weight must be >= width and multiples of 8 (ld_hidden=%lld, ld_weight=%lld)", (long long)ld_hidden, (long long)ld_weight);
    QLESS_REQUIRE(grad_hidden == nullptr || (aligned(grad_hidden, 16) && ld_grad_hidden >= width && ld_grad_hidden % 8 == 0), QLESS_ERR_INVALID_ARG,
                  "grad_hidden must be 16-byte aligned, ld_grad_hidden >= width and a multiple of 8 (ld_grad_hidden=%lld)", (long long)ld_grad_hidden);
    const LossPlan pl = plan_loss(tokens, width, vocab, grad_hidden != nullptr, grad_weight != nullptr);
    QLESS_REQUIRE(workspace != nullptr && aligned(workspace, 256), QLESS_ERR_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
    QLESS_REQUIRE(workspace_bytes >= pl.total, QLESS_ERR_WORKSPACE, "workspace too small: %zu bytes given, %zu needed", workspace_bytes, pl.total);
    unsigned int* flag = timeout_flag_ptr();
    QLESS_REQUIRE(flag != nullptr, QLESS_ERR_CUDA, "cannot resolve the device timeout flag");
    LossArgs a;
    a.hidden = hidden; a.weight = weight; a.labels = labels; a.token_weight = token_weight;
    a.T = tokens; a.ld_hidden = ld_hidden; a.ld_weight = ld_weight; a.ld_grad_hidden = ld_grad_hidden; a.ld_grad_weight = ld_grad_weight;
    a.width = width; a.vocab = vocab; a.loss = loss; a.grad_hidden = grad_hidden; a.grad_weight = grad_weight;
    return launch_loss(a, pl, reinterpret_cast<uint8_t*>(workspace), flag, st);
}

}  // extern "C"
