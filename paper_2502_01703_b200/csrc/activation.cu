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
// independent loads in flight (8 instead of 4: 171 -> 159 us and 166 -> 151 us for 65521 x 4112 bf16). Only the last group of a row may be short. Rows whose start or stride is not a multiple of the
// vector width are read element by element (same kernel, VEC = false).
#include "qless_kernels.h"

namespace qless {

namespace {

constexpr int THREADS = 256;
constexpr int LANE_CH = 8;                  // channels per lane
constexpr int SEG = 32 * LANE_CH;           // channels per warp and token
constexpr int UNROLL = 8;                   // tokens per warp and step

struct ActParams {
    int64_t tokens, ld_x, ld_codes, ld_scales;
    int32_t width, group, segments;
    int64_t units;                          // (token octets) x segments
};

__device__ __forceinline__ float max_nan_abs(float a, float b)      // max(a, |b|), NaN if either is
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const __nv_bfloat162 z = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&z);
}

// Eight channels of a lane as loaded: 8 words of fp32, or 4 words of two bf16.
template <typename T> struct Raw;
template <> struct Raw<float> {
    uint32_t w[8];
    __device__ __forceinline__ void load(const float* p)
    {
        const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p)), b = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    }
    __device__ __forceinline__ void set(int i, float v) { w[i] = __float_as_uint(v); }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(w[i]); }
    static constexpr int WORDS = 8;
    static __device__ __forceinline__ float read(const float* p) { return *p; }
    static __device__ __forceinline__ void store(float* p, const float (&v)[LANE_CH])
    {
        __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
        __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
    }
    static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
};
template <> struct Raw<__nv_bfloat16> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const __nv_bfloat16* p)
    {
        const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p));
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
    }
    __device__ __forceinline__ void set(int i, float v)      // v is a bf16 value; the words start at 0
    {
        w[i >> 1] |= (i & 1) ? (__float_as_uint(v) & 0xFFFF0000u) : (__float_as_uint(v) >> 16);
    }
    __device__ __forceinline__ float get(int i) const { return (i & 1) ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]); }
    static constexpr int WORDS = 4;
    static __device__ __forceinline__ float read(const __nv_bfloat16* p) { return __bfloat162float(*p); }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&v)[LANE_CH])
    {
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])));
    }
    static __device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
};

// The division by a run-time number of segments is done once per warp; the loop steps (octet, segment) by constant amounts.
struct Walk {
    int64_t octet; int32_t seg; int64_t dq; int32_t ds;
    __device__ __forceinline__ Walk(const ActParams& p)
    {
        const int64_t first = (int64_t)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5), step = (int64_t)gridDim.x * (THREADS / 32);
        octet = first / p.segments; seg = (int32_t)(first - octet * p.segments);
        dq = step / p.segments; ds = (int32_t)(step - dq * p.segments);
    }
    __device__ __forceinline__ void next(const ActParams& p)
    {
        octet += dq; seg += ds;
        if (seg >= p.segments) { seg -= p.segments; ++octet; }
    }
};

template <typename T, bool VEC, int GROUP>
__global__ void __launch_bounds__(THREADS) activation_quantize_kernel(const T* __restrict__ x, int8_t* __restrict__ codes,
                                                                      uint8_t* __restrict__ scales, const ActParams p)
{
    constexpr int LANES = GROUP / LANE_CH;                              // neighbouring lanes that share a step
    const int lane = threadIdx.x & 31;
    const int64_t octets = (p.tokens + UNROLL - 1) / UNROLL;
    ahead_release();
    ahead_wait();
    for (Walk u(p); u.octet < octets; u.next(p)) {
        const int c = u.seg * SEG + lane * LANE_CH;
        const int have = min(LANE_CH, p.width - c);                     // channels of this lane (<= 0: none)
        Raw<T> r[UNROLL];
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            const int64_t t = u.octet * UNROLL + k;
#pragma unroll
            for (int i = 0; i < Raw<T>::WORDS; ++i) r[k].w[i] = 0u;
            if (t < p.tokens) {
                const T* src = x + t * p.ld_x + c;
                if (VEC && have == LANE_CH) r[k].load(src);
                else {
#pragma unroll
                    for (int i = 0; i < LANE_CH; ++i) if (i < have) r[k].set(i, Raw<T>::read(src + i));
                }
            }
        }
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            const int64_t t = u.octet * UNROLL + k;
            float a = 0.0f;
#pragma unroll
            for (int i = 0; i < LANE_CH; ++i) a = max_nan_abs(a, r[k].get(i));
#pragma unroll
            for (int s = 1; s < LANES; s <<= 1) a = max_nan_abs(a, __shfl_xor_sync(0xFFFFFFFFu, a, s));
            const uint32_t top = __float_as_uint(a);
            // a = 1.m * 2^E: 127 * 2^(E-6) covers it unless 1.m > 127/64
            int e = (int)(top >> 23) - 127 - 6 + ((top & 0x7FFFFFu) > 0x7E0000u ? 1 : 0);
            const bool over = e > 121;                                  // above 127 * 2^121 (or not finite)
            e = max(-120, min(121, e));
            const bool finite = top < 0x7F800000u;
            const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
            // Adding 1.5 * 2^23 rounds to a whole number, half to even, and leaves it in two's complement in the low bits (the product
            // is exact, so the fused multiply-add rounds once).
            uint32_t q[LANE_CH];
#pragma unroll
            for (int i = 0; i < LANE_CH; ++i) q[i] = __float_as_uint(fmaf(r[k].get(i), inv, 12582912.0f));
            if (over) {
#pragma unroll
                for (int i = 0; i < LANE_CH; ++i) q[i] = finite ? (uint32_t)max(-127, min(127, __float2int_rn(r[k].get(i) * inv))) : 0u;
            }
            const uint32_t w0 = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
            const uint32_t w1 = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
            if (t < p.tokens && have > 0) {
                int8_t* dst = codes + t * p.ld_codes + c;
                if (VEC && have == LANE_CH) *reinterpret_cast<uint2*>(dst) = make_uint2(w0, w1);
                else {
#pragma unroll
                    for (int i = 0; i < LANE_CH; ++i) if (i < have) dst[i] = (int8_t)((i < 4 ? w0 : w1) >> (8 * (i & 3)));
                }
                if (lane % LANES == 0) scales[t * p.ld_scales + c / GROUP] = finite ? (uint8_t)(e + 127) : (uint8_t)0xFF;
            }
        }
    }
}

template <typename T, bool VEC, int GROUP>
__global__ void __launch_bounds__(THREADS) activation_dequantize_kernel(const int8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                                        T* __restrict__ out, const ActParams p)
{
    const int lane = threadIdx.x & 31;
    const int64_t octets = (p.tokens + UNROLL - 1) / UNROLL;
    ahead_release();
    ahead_wait();
    for (Walk u(p); u.octet < octets; u.next(p)) {
        const int c = u.seg * SEG + lane * LANE_CH;
        const int have = min(LANE_CH, p.width - c);
        if (have <= 0) continue;
        uint32_t w[UNROLL][2], step[UNROLL];
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            const int64_t t = u.octet * UNROLL + k;
            w[k][0] = w[k][1] = step[k] = 0u;
            if (t < p.tokens) {
                const int8_t* src = codes + t * p.ld_codes + c;
                step[k] = scales[t * p.ld_scales + c / GROUP];
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
            const int64_t t = u.octet * UNROLL + k;
            if (t >= p.tokens) continue;
            const float s = __uint_as_float(step[k] == 0xFFu ? 0x7FC00000u : step[k] << 23);      // NaN, or 2^(byte - 127)
            // The byte code + 128 under the bits of 2^23 is the number 2^23 + 128 + code (integer conversions run at a quarter of the rate).
            float v[LANE_CH];
#pragma unroll
            for (int i = 0; i < LANE_CH; ++i)
                v[i] = (__uint_as_float(__byte_perm(w[k][i >> 2] ^ 0x80808080u, 0x4B000000u, 0x7440 | (i & 3))) - 8388736.0f) * s;
            T* dst = out + t * p.ld_x + c;
            if (VEC && have == LANE_CH) Raw<T>::store(dst, v);
            else {
#pragma unroll
                for (int i = 0; i < LANE_CH; ++i) if (i < have) Raw<T>::put(dst + i, v[i]);
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

unsigned blocks_of(const ActParams& p) { return (unsigned)((p.units + THREADS / 32 - 1) / (THREADS / 32)); }
// Quantising, a block that stays saves its set-up (159 us against 166 us for 65521 x 4112 bf16); restoring, blocks that come and go
// spread the reads and writes better (138 us against 151 us).
unsigned staying_blocks_of(const ActParams& p)
{
    const unsigned blocks = blocks_of(p), most = (unsigned)sm_count() * 8;
    return blocks < most ? blocks : most;
}

bool vectors_fit(const void* x, int64_t ld_x, size_t esize, const void* codes, int64_t ld_codes)
{
    return reinterpret_cast<uintptr_t>(x) % 16 == 0 && (ld_x * esize) % 16 == 0 && reinterpret_cast<uintptr_t>(codes) % 8 == 0 && ld_codes % 8 == 0;
}

template <typename T, bool VEC>
cudaError_t quantize_group(const void* x, int8_t* codes, uint8_t* scales, const ActParams& p, cudaStream_t st)
{
    const T* src = reinterpret_cast<const T*>(x);
    const unsigned grid = staying_blocks_of(p);
    cudaError_t e;
    if (p.group == 32) e = launch_ahead(activation_quantize_kernel<T, VEC, 32>, dim3(grid), dim3(THREADS), 0, st, src, codes, scales, p);
    else if (p.group == 64) e = launch_ahead(activation_quantize_kernel<T, VEC, 64>, dim3(grid), dim3(THREADS), 0, st, src, codes, scales, p);
    else e = launch_ahead(activation_quantize_kernel<T, VEC, 128>, dim3(grid), dim3(THREADS), 0, st, src, codes, scales, p);
    return e;
}
template <typename T, bool VEC>
cudaError_t dequantize_group(const int8_t* codes, const uint8_t* scales, void* out, const ActParams& p, cudaStream_t st)
{
    T* dst = reinterpret_cast<T*>(out);
    const unsigned grid = blocks_of(p);
    cudaError_t e;
    if (p.group == 32) e = launch_ahead(activation_dequantize_kernel<T, VEC, 32>, dim3(grid), dim3(THREADS), 0, st, codes, scales, dst, p);
    else if (p.group == 64) e = launch_ahead(activation_dequantize_kernel<T, VEC, 64>, dim3(grid), dim3(THREADS), 0, st, codes, scales, dst, p);
    else e = launch_ahead(activation_dequantize_kernel<T, VEC, 128>, dim3(grid), dim3(THREADS), 0, st, codes, scales, dst, p);
    return e;
}

}  // namespace

cudaError_t launch_activation_quantize(const void* x, qless_dtype dtype, int64_t tokens, int32_t width, int64_t ld_x, int32_t group,
                                       int8_t* codes, int64_t ld_codes, uint8_t* scales, int64_t ld_scales, cudaStream_t st)
{
    const ActParams p = make_params(tokens, width, group, ld_x, ld_codes, ld_scales);
    const bool vec = vectors_fit(x, ld_x, dtype == QLESS_F32 ? 4 : 2, codes, ld_codes);
    count_launches(1);
    if (dtype == QLESS_F32) return vec ? quantize_group<float, true>(x, codes, scales, p, st) : quantize_group<float, false>(x, codes, scales, p, st);
    return vec ? quantize_group<__nv_bfloat16, true>(x, codes, scales, p, st) : quantize_group<__nv_bfloat16, false>(x, codes, scales, p, st);
}

cudaError_t launch_activation_dequantize(const int8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t ld_scales, int64_t tokens,
                                         int32_t width, int32_t group, void* out, qless_dtype dtype, int64_t ld_out, cudaStream_t st)
{
    const ActParams p = make_params(tokens, width, group, ld_out, ld_codes, ld_scales);
    const bool vec = vectors_fit(out, ld_out, dtype == QLESS_F32 ? 4 : 2, codes, ld_codes);
    count_launches(1);
    if (dtype == QLESS_F32) return vec ? dequantize_group<float, true>(codes, scales, out, p, st) : dequantize_group<float, false>(codes, scales, out, p, st);
    return vec ? dequantize_group<__nv_bfloat16, true>(codes, scales, out, p, st) : dequantize_group<__nv_bfloat16, false>(codes, scales, out, p, st);
}

}  // namespace qless
