// 8-bit activation checkpoints: groups of g = 32, 64 or 128 channels of a token share one power-of-two step.
//
//   a = max |x| over the group, e = the smallest integer with a <= 127 * 2^e, kept within [-120, 121];
//   code = round_half_even(x * 2^-e), stored step byte = e + 127 (0xFF: the group holds an infinity or a NaN).
//
// The step is a power of two because the codes then stand for values that bf16 holds exactly (8 significant bits), so the
// backward pass can hand them to a bf16 tensor-core product without rounding them a second time; x * 2^-e is exact, so the
// codes are the same on every machine. It costs up to one bit against a / 127 as the step, which the small groups more than
// make up for: a row-wide step would be set by the row's few large channels.
//
// Bound by HBM: esize + 1 + 1/g bytes per element each way. A warp owns 256 channels (8 per lane: one 16-byte load of bf16,
// two of fp32; g / 8 neighbouring lanes form a group) and UNROLL tokens at a time, so that every lane has that many
// independent loads in flight. Only the last group of a row may be short. Rows whose start or stride is not a multiple of the
// vector width are read element by element (same kernel, VEC = false).
#include "qless_kernels.h"

namespace qless {

namespace {

constexpr int THREADS = 256;
constexpr int LANE_CH = 8;                  // channels per lane
constexpr int SEG = 32 * LANE_CH;           // channels per warp and token
constexpr int UNROLL = 4;                   // tokens per warp and step

template <typename T> struct Chunk;
template <> struct Chunk<float> {
    static __device__ __forceinline__ void load(const float* p, float (&v)[LANE_CH])
    {
        const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    static __device__ __forceinline__ float one(const float* p) { return *p; }
    static __device__ __forceinline__ void store(float* p, const float (&v)[LANE_CH])
    {
        __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
        __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
    }
    static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
};
template <> struct Chunk<__nv_bfloat16> {
    static __device__ __forceinline__ void load(const __nv_bfloat16* p, float (&v)[LANE_CH])
    {
        const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p));
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
    static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&v)[LANE_CH])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 z = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&z);
        }
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
    }
    static __device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
};

struct ActParams {
    int64_t tokens, ld_x, ld_codes, ld_scales;
    int32_t width, group, segments;
    int64_t units;                          // (token quads) x segments
};

template <typename T, bool VEC>
__global__ void __launch_bounds__(THREADS) activation_quantize_kernel(const T* __restrict__ x, int8_t* __restrict__ codes,
                                                                      uint8_t* __restrict__ scales, const ActParams p)
{
    const int lane = threadIdx.x & 31;
    const int lanes_per_group = p.group / LANE_CH;
    const int64_t warps = (int64_t)gridDim.x * (THREADS / 32);
    for (int64_t u = (int64_t)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5); u < p.units; u += warps) {
        const int64_t quad = u / p.segments;
        const int c = (int)(u - quad * p.segments) * SEG + lane * LANE_CH;
        const int have = min(LANE_CH, p.width - c);                     // channels of this lane (<= 0: none)
        float v[UNROLL][LANE_CH];
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            const int64_t t = quad * UNROLL + k;
#pragma unroll
            for (int i = 0; i < LANE_CH; ++i) v[k][i] = 0.0f;
            if (t < p.tokens) {
                const T* src = x + t * p.ld_x + c;
                if (VEC && have == LANE_CH) Chunk<T>::load(src, v[k]);
                else {
#pragma unroll
                    for (int i = 0; i < LANE_CH; ++i) if (i < have) v[k][i] = Chunk<T>::one(src + i);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            const int64_t t = quad * UNROLL + k;
            uint32_t top = 0;                                           // |x| as bits: ordered, NaN above infinity above the rest
#pragma unroll
            for (int i = 0; i < LANE_CH; ++i) top = max(top, __float_as_uint(v[k][i]) & 0x7FFFFFFFu);
            for (int s = 1; s < lanes_per_group; s <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
            // a = 1.m * 2^E: 127 * 2^(E-6) covers it unless 1.m > 127/64
            int e = (int)(top >> 23) - 127 - 6 + ((top & 0x7FFFFFu) > 0x7E0000u ? 1 : 0);
            e = max(-120, min(121, e));
            const bool finite = top < 0x7F800000u;
            const float inv = finite ? __uint_as_float((uint32_t)(127 - e) << 23) : 0.0f;
            uint32_t w[2] = {0u, 0u};
#pragma unroll
            for (int i = 0; i < LANE_CH; ++i) {
                // the upper clamp acts only where a lies above 127 * 2^121, the largest value that the codes can stand for
                const int q = finite ? max(-127, min(127, __float2int_rn(v[k][i] * inv))) : 0;
                w[i >> 2] |= ((uint32_t)q & 0xFFu) << (8 * (i & 3));
            }
            if (t < p.tokens && have > 0) {
                int8_t* dst = codes + t * p.ld_codes + c;
                if (VEC && have == LANE_CH) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
                else {
#pragma unroll
                    for (int i = 0; i < LANE_CH; ++i) if (i < have) dst[i] = (int8_t)(w[i >> 2] >> (8 * (i & 3)));
                }
                if (lane % lanes_per_group == 0) scales[t * p.ld_scales + c / p.group] = finite ? (uint8_t)(e + 127) : (uint8_t)0xFF;
            }
        }
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(THREADS) activation_dequantize_kernel(const int8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                                        T* __restrict__ out, const ActParams p)
{
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * (THREADS / 32);
    for (int64_t u = (int64_t)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5); u < p.units; u += warps) {
        const int64_t quad = u / p.segments;
        const int c = (int)(u - quad * p.segments) * SEG + lane * LANE_CH;
        const int have = min(LANE_CH, p.width - c);
        if (have <= 0) continue;
        uint32_t w[UNROLL][2], step[UNROLL];
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            const int64_t t = quad * UNROLL + k;
            w[k][0] = w[k][1] = step[k] = 0u;
            if (t < p.tokens) {
                const int8_t* src = codes + t * p.ld_codes + c;
                step[k] = scales[t * p.ld_scales + c / p.group];
                if (VEC && have == LANE_CH) {
                    const uint2 a = *reinterpret_cast<const uint2*>(src);
                    w[k][0] = a.x; w[k][1] = a.y;
                } else {
#pragma unroll
                    for (int i = 0; i < LANE_CH; ++i) if (i < have) w[k][i >> 2] |= ((uint32_t)(uint8_t)src[i]) << (8 * (i & 3));
                }
            }
        }
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            const int64_t t = quad * UNROLL + k;
            if (t >= p.tokens) continue;
            const float s = __uint_as_float(step[k] == 0xFFu ? 0x7FC00000u : step[k] << 23);      // NaN, or 2^(byte - 127)
            float v[LANE_CH];
#pragma unroll
            for (int i = 0; i < LANE_CH; ++i) v[i] = (float)(int8_t)(w[k][i >> 2] >> (8 * (i & 3))) * s;
            T* dst = out + t * p.ld_x + c;
            if (VEC && have == LANE_CH) Chunk<T>::store(dst, v);
            else {
#pragma unroll
                for (int i = 0; i < LANE_CH; ++i) if (i < have) Chunk<T>::put(dst + i, v[i]);
            }
        }
    }
}

ActParams make_params(int64_t tokens, int32_t width, int32_t group, int64_t ld_x, int64_t ld_codes, int64_t ld_scales)
{
    ActParams p;
    p.tokens = tokens; p.ld_x = ld_x; p.ld_codes = ld_codes; p.ld_scales = ld_scales;
    p.width = width; p.group = group; p.segments = (width + SEG - 1) / SEG;
    p.units = (tokens + UNROLL - 1) / UNROLL * p.segments;
    return p;
}

unsigned grid_for(const ActParams& p)
{
    const int64_t blocks = (p.units + THREADS / 32 - 1) / (THREADS / 32);
    const int64_t most = (int64_t)sm_count() * 8;
    return (unsigned)(blocks < most ? blocks : most);
}

bool vectors_fit(const void* x, int64_t ld_x, size_t esize, const void* codes, int64_t ld_codes)
{
    return reinterpret_cast<uintptr_t>(x) % 16 == 0 && (ld_x * esize) % 16 == 0 && reinterpret_cast<uintptr_t>(codes) % 8 == 0 && ld_codes % 8 == 0;
}

}  // namespace

cudaError_t launch_activation_quantize(const void* x, qless_dtype dtype, int64_t tokens, int32_t width, int64_t ld_x, int32_t group,
                                       int8_t* codes, int64_t ld_codes, uint8_t* scales, int64_t ld_scales, cudaStream_t st)
{
    const ActParams p = make_params(tokens, width, group, ld_x, ld_codes, ld_scales);
    const bool vec = vectors_fit(x, ld_x, dtype == QLESS_F32 ? 4 : 2, codes, ld_codes);
    const unsigned grid = grid_for(p);
    if (dtype == QLESS_F32) {
        const float* src = reinterpret_cast<const float*>(x);
        if (vec) activation_quantize_kernel<float, true><<<grid, THREADS, 0, st>>>(src, codes, scales, p);
        else activation_quantize_kernel<float, false><<<grid, THREADS, 0, st>>>(src, codes, scales, p);
    } else {
        const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(x);
        if (vec) activation_quantize_kernel<__nv_bfloat16, true><<<grid, THREADS, 0, st>>>(src, codes, scales, p);
        else activation_quantize_kernel<__nv_bfloat16, false><<<grid, THREADS, 0, st>>>(src, codes, scales, p);
    }
    count_launches(1);
    return cudaGetLastError();
}

cudaError_t launch_activation_dequantize(const int8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t ld_scales, int64_t tokens,
                                         int32_t width, int32_t group, void* out, qless_dtype dtype, int64_t ld_out, cudaStream_t st)
{
    const ActParams p = make_params(tokens, width, group, ld_out, ld_codes, ld_scales);
    const bool vec = vectors_fit(out, ld_out, dtype == QLESS_F32 ? 4 : 2, codes, ld_codes);
    const unsigned grid = grid_for(p);
    if (dtype == QLESS_F32) {
        float* dst = reinterpret_cast<float*>(out);
        if (vec) activation_dequantize_kernel<float, true><<<grid, THREADS, 0, st>>>(codes, scales, dst, p);
        else activation_dequantize_kernel<float, false><<<grid, THREADS, 0, st>>>(codes, scales, dst, p);
    } else {
        __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(out);
        if (vec) activation_dequantize_kernel<__nv_bfloat16, true><<<grid, THREADS, 0, st>>>(codes, scales, dst, p);
        else activation_dequantize_kernel<__nv_bfloat16, false><<<grid, THREADS, 0, st>>>(codes, scales, dst, p);
    }
    count_launches(1);
    return cudaGetLastError();
}

}  // namespace qless
