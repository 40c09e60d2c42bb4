// Layer normalisation of the rows of a matrix, forward and backward (with `center` off: by the root mean square alone).
//
//   mu = mean x (0 without centring),  r = 1 / sqrt(mean (x - mu)^2 + eps),  xh = (x - mu) r,  y = xh w + b
//   g = w dy;  dx = r (g - mean g - xh mean(g xh)) (no mean g without centring);  dw = sum_t dy xh;  db = sum_t dy
//
// Bound: bytes (forward: x read, y written; backward: x and dy read, dx written; a few operations an element). A row is read once: its
// values stay in the registers of the threads that share it (32 values a thread, as 16-byte vectors where rows are aligned, else element by
// element with neighbouring lanes on neighbouring elements), and the moments are taken from them in two steps, mean and then squares
// of the differences, so that a mean far from zero costs no digits. 32, 128, 256 or 512 threads share a row: the fewest that hold it.
// dw and db: blocks that walk over the rows keep their columns' sums in registers and leave one row of fp32 sums each, which a second
// kernel adds in a fixed order (no atomics: the same inputs give the same bits).
#include "qless_kernels.h"

namespace qless {

namespace {

constexpr int VALUES = 32;                  // of a row, held by one thread
constexpr int ROOM_BLOCK = 256;             // threads of a block, where no more are needed for one row

template <typename T> struct Elem;
template <> struct Elem<float> {
    static constexpr int VEC = 4;
    static __device__ __forceinline__ void unpack(const uint4& u, float* v)
    {
        v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 pack(const float* v)
    {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
    static __device__ __forceinline__ float get(const float* p) { return *p; }
    static __device__ __forceinline__ void put(float* p, float x) { *p = x; }
};
template <> struct Elem<__nv_bfloat16> {
    static constexpr int VEC = 8;
    static __device__ __forceinline__ void unpack(const uint4& u, float* v)
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) { v[2 * k] = __uint_as_float(w[k] << 16); v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u); }
    }
    static __device__ __forceinline__ uint4 pack(const float* v)
    {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __nv_bfloat162 z = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
            w[k] = *reinterpret_cast<const uint32_t*>(&z);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float get(const __nv_bfloat16* p) { return __bfloat162float(*p); }
    static __device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
};

// A thread's values of a row: value [n][e] is element (n * share + rank) * V + e.
template <typename T, int V>
__device__ __forceinline__ void load_row(const T* row, int width, int rank, int share, float (&v)[VALUES])
{
    constexpr int N = VALUES / V;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int c = (n * share + rank) * V;
        if constexpr (V == 1) {
            v[n] = c < width ? Elem<T>::get(row + c) : 0.0f;
        } else {
            uint4 u = make_uint4(0u, 0u, 0u, 0u);
            if (c < width) u = __ldg(reinterpret_cast<const uint4*>(row + c));
            Elem<T>::unpack(u, v + n * V);
        }
    }
}
// V parameters from element c on, whatever their type (c < width).
template <typename P, int V>
__device__ __forceinline__ void load_params(const P* p, int c, float (&v)[V])
{
    if constexpr (V == 1) {
        v[0] = Elem<P>::get(p + c);
    } else {
        constexpr int PV = Elem<P>::VEC < V ? Elem<P>::VEC : V;
        if constexpr (PV == Elem<P>::VEC) {
#pragma unroll
            for (int k = 0; k < V; k += PV) Elem<P>::unpack(__ldg(reinterpret_cast<const uint4*>(p + c + k)), v + k);
        } else {                                             // four bf16 parameters beside four fp32 values
            const uint2 u = __ldg(reinterpret_cast<const uint2*>(p + c));
            v[0] = __uint_as_float(u.x << 16); v[1] = __uint_as_float(u.x & 0xFFFF0000u);
            v[2] = __uint_as_float(u.y << 16); v[3] = __uint_as_float(u.y & 0xFFFF0000u);
        }
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[V])
{
    if constexpr (V == 1) Elem<T>::put(p, v[0]);
    else *reinterpret_cast<uint4*>(p) = Elem<T>::pack(v);
}

// Sums of K numbers over the threads that share a row (a warp, or the whole block), in every one of them. `room` alternates between two halves,
// so that one barrier per call is enough: a half is written again only behind the barrier of the call after.
template <int K>
__device__ __forceinline__ void row_sum(float (&x)[K], int share, float (*room)[16][2], int& turn)
{
#pragma unroll
    for (int s = 16; s > 0; s >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) x[k] += __shfl_xor_sync(0xFFFFFFFFu, x[k], s);
    if (share == 32) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) room[turn][warp][k] = x[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        x[k] = lane < (share >> 5) ? room[turn][lane][k] : 0.0f;
#pragma unroll
        for (int s = 16; s > 0; s >>= 1) x[k] += __shfl_xor_sync(0xFFFFFFFFu, x[k], s);
    }
    turn ^= 1;
}

struct NormParams {
    const void* x; const void* dy; const void* weight; const void* bias;
    void* out;                              // y, or dx
    float* mean; float* rstd;               // written by the forward kernel (NULL: not wanted), read by the other (mean NULL: 0)
    float* part;                            // [workers][2][width]: sums of dw and db
    int64_t tokens, ld_x, ld_dy, ld_out;
    int32_t width, share, center;
    float eps;
};

template <typename T, typename P, int V>
__global__ void __launch_bounds__(512) norm_forward_kernel(const NormParams p)
{
    __shared__ float room[2][16][2];
    ahead_wait();
    ahead_release();
    int turn = 0;
    const int share = p.share, rank = threadIdx.x % share;
    const int64_t t = (int64_t)blockIdx.x * (blockDim.x / share) + threadIdx.x / share;
    if (t >= p.tokens) return;                               // whole warps: a block of one row has it
    float v[VALUES];
    load_row<T, V>(reinterpret_cast<const T*>(p.x) + t * p.ld_x, p.width, rank, share, v);
    const float inv = 1.0f / (float)p.width;
    float mu = 0.0f;
    if (p.center) {
        float s[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < VALUES; ++k) s[0] += v[k];       // places behind the row hold 0
        row_sum<1>(s, share, room, turn);
        mu = s[0] * inv;
    }
    float s[1] = {0.0f};
#pragma unroll
    for (int n = 0; n < VALUES / V; ++n) {
        if ((n * share + rank) * V >= p.width) break;
#pragma unroll
        for (int e = 0; e < V; ++e) { v[n * V + e] -= mu; s[0] = fmaf(v[n * V + e], v[n * V + e], s[0]); }
    }
    row_sum<1>(s, share, room, turn);
    const float r = rsqrtf(fmaf(s[0], inv, p.eps));
    if (rank == 0) {
        if (p.mean != nullptr) p.mean[t] = mu;
        if (p.rstd != nullptr) p.rstd[t] = r;
    }
    T* out = reinterpret_cast<T*>(p.out) + t * p.ld_out;
#pragma unroll
    for (int n = 0; n < VALUES / V; ++n) {
        const int c = (n * share + rank) * V;
        if (c >= p.width) break;
        float w[V], b[V], y[V];
        load_params<P, V>(reinterpret_cast<const P*>(p.weight), c, w);
        if (p.bias != nullptr) load_params<P, V>(reinterpret_cast<const P*>(p.bias), c, b);
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = p.bias != nullptr ? fmaf(v[n * V + e] * r, w[e], b[e]) : v[n * V + e] * r * w[e];
        store_vec<T, V>(out + c, y);
    }
}

// A worker (the threads that share a row) takes every workers-th row; SUMS: it keeps its columns' sums and leaves them in part.
template <typename T, typename P, int V, bool SUMS, int BLOCK>
__global__ void __launch_bounds__(BLOCK) norm_backward_kernel(const NormParams p)
{
    __shared__ float room[2][16][2];
    ahead_wait();
    ahead_release();
    int turn = 0;
    const int share = p.share, rank = threadIdx.x % share, per = blockDim.x / share;
    const int64_t worker = (int64_t)blockIdx.x * per + threadIdx.x / share, workers = (int64_t)gridDim.x * per;
    const float inv = 1.0f / (float)p.width;
    float sw[SUMS ? VALUES : 1], sb[SUMS ? VALUES : 1];
    if (SUMS) {
#pragma unroll
        for (int k = 0; k < VALUES; ++k) sw[k] = sb[k] = 0.0f;
    }
    for (int64_t t = worker; t < p.tokens; t += workers) {   // (a block of one worker: the same trips for all of its threads)
        float x[VALUES], g[VALUES];
        load_row<T, V>(reinterpret_cast<const T*>(p.x) + t * p.ld_x, p.width, rank, share, x);
        load_row<T, V>(reinterpret_cast<const T*>(p.dy) + t * p.ld_dy, p.width, rank, share, g);
        const float mu = p.mean != nullptr ? p.mean[t] : 0.0f, r = p.rstd[t];
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int n = 0; n < VALUES / V; ++n) {
            const int c = (n * share + rank) * V;
            if (c >= p.width) break;
            float w[V];
            load_params<P, V>(reinterpret_cast<const P*>(p.weight), c, w);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int k = n * V + e;
                x[k] = (x[k] - mu) * r;
                if (SUMS) { sw[k] = fmaf(g[k], x[k], sw[k]); sb[k] += g[k]; }
                g[k] *= w[e];
                s[0] += g[k];
                s[1] = fmaf(g[k], x[k], s[1]);
            }
        }
        row_sum<2>(s, share, room, turn);
        const float m = p.center ? s[0] * inv : 0.0f, along = s[1] * inv;
        T* out = reinterpret_cast<T*>(p.out) + t * p.ld_out;
#pragma unroll
        for (int n = 0; n < VALUES / V; ++n) {
            const int c = (n * share + rank) * V;
            if (c >= p.width) break;
            float d[V];
#pragma unroll
            for (int e = 0; e < V; ++e) d[e] = (g[n * V + e] - m - x[n * V + e] * along) * r;
            store_vec<T, V>(out + c, d);
        }
    }
    if (SUMS) {
        float* dst = p.part + worker * 2 * p.width;
#pragma unroll
        for (int n = 0; n < VALUES / V; ++n) {
            const int c = (n * share + rank) * V;
            if (c >= p.width) break;
#pragma unroll
            for (int e = 0; e < V; ++e) { dst[c + e] = sw[n * V + e]; dst[p.width + c + e] = sb[n * V + e]; }
        }
    }
}

// dw and db from the workers' sums: a block has 32 columns (of dw, then of db), its 32 warps every 32nd worker each, joined in order.
template <typename P>
__global__ void __launch_bounds__(1024) norm_join_kernel(const float* __restrict__ part, int64_t workers, int32_t width, P* dw, P* db)
{
    __shared__ float sums[32][33];
    ahead_wait();
    ahead_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int groups = (width + 31) / 32, which = blockIdx.x / groups, c = (blockIdx.x - which * groups) * 32 + lane;
    float s = 0.0f;
    if (c < width)
        for (int64_t k = warp; k < workers; k += 32) s += part[(2 * k + which) * width + c];
    sums[warp][lane] = s;
    __syncthreads();
    if (warp > 0 || c >= width) return;
    s = 0.0f;
#pragma unroll
    for (int k = 0; k < 32; ++k) s += sums[k][lane];
    P* dst = which ? db : dw;
    if (dst != nullptr) Elem<P>::put(dst + c, s);
}

bool vectors(const void* p, int64_t ld, int elem)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * elem % 16 == 0;
}

}  // namespace

NormPlan plan_norm(int64_t tokens, int32_t width, bool sums)
{
    NormPlan pl;
    pl.share = width <= 32 * VALUES ? 32 : width <= 128 * VALUES ? 128 : width <= 256 * VALUES ? 256 : 512;
    pl.block = pl.share < ROOM_BLOCK ? ROOM_BLOCK : pl.share;
    if (pl.share == 128) pl.block = 128;                     // a block's barriers are for one row
    const int per = pl.block / pl.share;
    const int64_t blocks = (tokens + per - 1) / per;
    // Workers that keep sums: as many as are resident (a thread needs up to 128 registers).
    const int64_t most = (int64_t)sm_count() * (pl.block == 128 ? 4 : pl.block == 256 ? 2 : 1);
    pl.blocks = sums && blocks > most ? most : blocks;
    pl.workers = pl.blocks * per;
    pl.total = sums ? align_up((size_t)pl.workers * 2 * width * 4, 256) + 256 : 256;
    return pl;
}

template <typename T, typename P>
static cudaError_t forward_of(const NormPlan& pl, const NormParams& p, bool vec, cudaStream_t st)
{
    const dim3 grid((unsigned)pl.blocks), block((unsigned)pl.block);
    return vec ? launch_ahead(norm_forward_kernel<T, P, Elem<T>::VEC>, grid, block, 0, st, p)
               : launch_ahead(norm_forward_kernel<T, P, 1>, grid, block, 0, st, p);
}

template <typename T, typename P>
static cudaError_t backward_of(const NormPlan& pl, const NormParams& p, bool vec, bool sums, cudaStream_t st)
{
    const dim3 grid((unsigned)pl.blocks), block((unsigned)pl.block);
    constexpr int V = Elem<T>::VEC;
    if (pl.block > 256) {                                    // 128 registers a thread instead of up to 255
        if (sums) return vec ? launch_ahead(norm_backward_kernel<T, P, V, true, 512>, grid, block, 0, st, p)
                             : launch_ahead(norm_backward_kernel<T, P, 1, true, 512>, grid, block, 0, st, p);
        return vec ? launch_ahead(norm_backward_kernel<T, P, V, false, 512>, grid, block, 0, st, p)
                   : launch_ahead(norm_backward_kernel<T, P, 1, false, 512>, grid, block, 0, st, p);
    }
    if (sums) return vec ? launch_ahead(norm_backward_kernel<T, P, V, true, 256>, grid, block, 0, st, p)
                         : launch_ahead(norm_backward_kernel<T, P, 1, true, 256>, grid, block, 0, st, p);
    return vec ? launch_ahead(norm_backward_kernel<T, P, V, false, 256>, grid, block, 0, st, p)
               : launch_ahead(norm_backward_kernel<T, P, 1, false, 256>, grid, block, 0, st, p);
}

qless_status launch_norm_forward(const NormArgs& a, cudaStream_t st)
{
    const NormPlan pl = plan_norm(a.tokens, a.width, false);
    const int es = a.dtype == QLESS_F32 ? 4 : 2, vec = 16 / es;
    const bool whole = a.width % vec == 0 && vectors(a.x, a.ld_x, es) && vectors(a.out, a.ld_out, es) && vectors(a.weight, 0, 1) &&
                       (a.bias == nullptr || vectors(a.bias, 0, 1));
    NormParams p{};
    p.x = a.x; p.weight = a.weight; p.bias = a.bias; p.out = a.out; p.mean = a.mean; p.rstd = a.rstd;
    p.tokens = a.tokens; p.ld_x = a.ld_x; p.ld_out = a.ld_out; p.width = a.width; p.share = pl.share; p.center = a.center; p.eps = a.eps;
    ProfileScope ps("layer_norm", st);
    if (a.dtype == QLESS_F32) {
        if (a.param_dtype == QLESS_F32) QLESS_CUDA_TRY((forward_of<float, float>(pl, p, whole, st)));
        else QLESS_CUDA_TRY((forward_of<float, __nv_bfloat16>(pl, p, whole, st)));
    } else {
        if (a.param_dtype == QLESS_F32) QLESS_CUDA_TRY((forward_of<__nv_bfloat16, float>(pl, p, whole, st)));
        else QLESS_CUDA_TRY((forward_of<__nv_bfloat16, __nv_bfloat16>(pl, p, whole, st)));
    }
    count_launches(1);
    return QLESS_OK;
}

qless_status launch_norm_backward(const NormArgs& a, uint8_t* ws, cudaStream_t st)
{
    const bool sums = a.grad_weight != nullptr || a.grad_bias != nullptr;
    const NormPlan pl = plan_norm(a.tokens, a.width, sums);
    const int es = a.dtype == QLESS_F32 ? 4 : 2, vec = 16 / es;
    const bool whole = a.width % vec == 0 && vectors(a.x, a.ld_x, es) && vectors(a.dy, a.ld_dy, es) && vectors(a.out, a.ld_out, es) && vectors(a.weight, 0, 1);
    NormParams p{};
    p.x = a.x; p.dy = a.dy; p.weight = a.weight; p.out = a.out; p.mean = a.center ? a.mean : nullptr; p.rstd = a.rstd; p.part = reinterpret_cast<float*>(ws);
    p.tokens = a.tokens; p.ld_x = a.ld_x; p.ld_dy = a.ld_dy; p.ld_out = a.ld_out; p.width = a.width; p.share = pl.share; p.center = a.center;
    { ProfileScope ps("layer_norm_backward", st);
      if (a.dtype == QLESS_F32) {
          if (a.param_dtype == QLESS_F32) QLESS_CUDA_TRY((backward_of<float, float>(pl, p, whole, sums, st)));
          else QLESS_CUDA_TRY((backward_of<float, __nv_bfloat16>(pl, p, whole, sums, st)));
      } else {
          if (a.param_dtype == QLESS_F32) QLESS_CUDA_TRY((backward_of<__nv_bfloat16, float>(pl, p, whole, sums, st)));
          else QLESS_CUDA_TRY((backward_of<__nv_bfloat16, __nv_bfloat16>(pl, p, whole, sums, st)));
      } }
    count_launches(1);
    if (sums) {
        ProfileScope ps("layer_norm_join", st);
        const dim3 grid((unsigned)(2 * ((a.width + 31) / 32)));
        const float* part = p.part;
        if (a.param_dtype == QLESS_F32)
            QLESS_CUDA_TRY(launch_ahead(norm_join_kernel<float>, grid, dim3(1024), 0, st, part, pl.workers, a.width, reinterpret_cast<float*>(a.grad_weight),
                                        reinterpret_cast<float*>(a.grad_bias)));
        else
            QLESS_CUDA_TRY(launch_ahead(norm_join_kernel<__nv_bfloat16>, grid, dim3(1024), 0, st, part, pl.workers, a.width,
                                        reinterpret_cast<__nv_bfloat16*>(a.grad_weight), reinterpret_cast<__nv_bfloat16*>(a.grad_bias)));
        count_launches(1);
    }
    return QLESS_OK;
}

}  // namespace qless
