// What the kernels of the gated feed-forward block share.
#pragma once

#include <type_traits>

#include "qless_kernels.h"
#include "tc_common.cuh"

namespace qless {
namespace ffn {

using namespace tc;

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const __nv_bfloat162 z = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&z);
}
__device__ __forceinline__ void pack_row32(const float (&v)[32], uint4 (&w)[4])
{
#pragma unroll
    for (int k = 0; k < 4; ++k)
        w[k] = make_uint4(pack_bf16(v[8 * k], v[8 * k + 1]), pack_bf16(v[8 * k + 2], v[8 * k + 3]), pack_bf16(v[8 * k + 4], v[8 * k + 5]),
                          pack_bf16(v[8 * k + 6], v[8 * k + 7]));
}
__device__ __forceinline__ void unpack8(const uint4& u, float* v)
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { v[2 * k] = __uint_as_float(w[k] << 16); v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u); }
}
__device__ __forceinline__ void unpack_row32(const uint4 (&w)[4], float (&v)[32])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) unpack8(w[k], v + 8 * k);
}
__device__ __forceinline__ void load_acc(uint32_t taddr, float (&v)[32])
{
    uint32_t raw[32];
    __syncwarp();                                            // (the load is a whole warp's; lanes may come from stores that some of them did not make)
    tmem_ld_x32(taddr, raw);
    tmem_wait_ld();
#pragma unroll
    for (int k = 0; k < 32; ++k) v[k] = __uint_as_float(raw[k]);
}

// a = act(g) and its derivative. SiLU: g s, s + g s (1 - s) with s = 1 / (1 + e^-g); GELU: g F(g), F(g) + g f(g) with the normal
// distribution F and its density f.
template <int ACT>
__device__ __forceinline__ void activation(float g, float& a, float& da)
{
    if constexpr (ACT == QLESS_SILU) {
        const float s = __fdividef(1.0f, 1.0f + __expf(-g));      // (g far below 0: 1 / infinity = 0)
        a = g == -INFINITY ? 0.0f : g * s;
        da = isinf(g) ? s : fmaf(a, 1.0f - s, s);
    } else {
        const float F = 0.5f * erfcf(-0.70710678118654752f * g), f = 0.39894228040143268f * __expf(-0.5f * g * g);
        a = g == -INFINITY ? 0.0f : g * F;
        da = isinf(g) ? F : fmaf(g, f, F);
    }
}

// What is done for many elements is written once for each activation: with the choice made for every element anew they would follow one another instead of
// overlapping (dg and du of a 256 x 256 tile took 60 thousand clocks so, four times the product's).
template <typename F>
__device__ __forceinline__ void by_activation(int act, F f)
{
    if (act == QLESS_SILU) f(std::integral_constant<int, QLESS_SILU>{});
    else f(std::integral_constant<int, QLESS_GELU>{});
}

// Few tokens (ffn_few.cu): the weights' rows or columns are the tile's rows, the tokens its columns, as many as fit. 4096 x 11008, forward and
// backward: 200 tokens 96 and 100 us, 256 tokens 105 and 110 us; on pairs of SMs (ffn.cu) 117 and 162, 118 and 162 us.
constexpr int FEW = 256;
inline bool few_tokens(int64_t tokens) { return tokens <= FEW; }
size_t few_workspace(int64_t tokens, int32_t width, int32_t inner, bool backward);
qless_status launch_few_forward(const FfnArgs& a, uint8_t* ws, unsigned int* timeout_word, cudaStream_t st);
// dg, du, dx, and h where `hidden` is not NULL ([tokens, inner])
qless_status launch_few_backward(const FfnArgs& a, __nv_bfloat16* hidden, uint8_t* ws, unsigned int* timeout_word, cudaStream_t st);

}  // namespace ffn
}  // namespace qless
