// Layer normalisation of the rows of a matrix, forward and backward (with `center` off: by the root mean square alone).
//
//   mu = mean x (0 without centring),  r = 1 / sqrt(mean (x - mu)^2 + eps),  xh = (x - mu) r,  y = xh w + b
//   g = w dy;  dx = r (g - mean g - xh mean(g xh)) (no mean g without centring);  dw = sum_t dy xh;  db = sum_t dy
//
// Bound: bytes (forward: x read, y written; backward: x and dy read, dx written; a few operations an element). A row is read once: its
// values stay in the registers of the threads that share it (32 values a thread, as 16-byte vectors where rows are aligned, else element by
// element with neighbouring lanes on neighbouring elements), and the moments are taken from them in two steps, mean and then squares
// of the differences, so that a mean far from zero costs no digits. 32, 128, 256 or 512 threads share a row: the fewest that hold it.
// dw and db: workers that walk over the rows keep their columns' sums in registers and leave one row of fp32 sums each, which a second
// kernel adds in a fixed order (no atomics: the same inputs give the same bits). With the sums there is no room to hold rows ahead in
// registers, and few warps an SM: aligned rows of up to 8192 values come through a ring in shared memory (norm_backward_ring_kernel).
#include "qless_kernels.h"
#include "tc_common.cuh"

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

// The same with the sums, rows brought ahead by bulk copies: every worker has a ring of `stages` places of a row of x and one of dy. A row is read
// from its place twice (for the two means, then for dx); the place is filled again behind the barrier of the next row's means, when every
// thread of the worker has left it.
struct RingParams {
    NormParams n;
    int32_t stages, row_bytes;
    unsigned int* timeout_word;
};

struct __align__(128) RingBars {
    uint64_t full[8][8];                    // [worker of the block][place]
    float room[8][2][8][2];                 // [worker][turn][warp][mean]
    uint32_t abort_flag;
};

template <typename T, typename P>
__global__ void __launch_bounds__(256, 2) norm_backward_ring_kernel(const RingParams q)
{
    using namespace tc;
    constexpr int V = Elem<T>::VEC;
    extern __shared__ __align__(128) uint8_t smem[];
    RingBars* bars = reinterpret_cast<RingBars*>(smem);
    auto& full = bars->full;
    auto& room = bars->room;
    const NormParams& p = q.n;
    const int share = p.share, rank = threadIdx.x % share, mine = threadIdx.x / share, per = 256 / share;
    const int lane = threadIdx.x & 31, warp_of = rank >> 5, warps = share >> 5;
    if (threadIdx.x == 0) {
        for (int i = 0; i < per; ++i) for (int s = 0; s < q.stages; ++s) mbar_init(smem_u32(&full[i][s]), 1);
        bars->abort_flag = 0;
        fence_barrier_init();
    }
    __syncthreads();
    ahead_wait();
    ahead_release();
    const int64_t worker = (int64_t)blockIdx.x * per + mine, workers = (int64_t)gridDim.x * per;
    uint8_t* ring = smem + sizeof(RingBars) + (size_t)mine * q.stages * 2 * q.row_bytes;
    auto bring = [&](int64_t t, int place) {                 // one thread
        const uint32_t bar = smem_u32(&full[mine][place]), dst = smem_u32(ring + (size_t)place * 2 * q.row_bytes);
        mbar_arrive_expect_tx(bar, 2 * q.row_bytes);
        bulk_load(dst, reinterpret_cast<const T*>(p.x) + t * p.ld_x, q.row_bytes, bar);
        bulk_load(dst + q.row_bytes, reinterpret_cast<const T*>(p.dy) + t * p.ld_dy, q.row_bytes, bar);
    };
    if (rank == 0)
        for (int s = 0; s < q.stages && worker + s * workers < p.tokens; ++s) bring(worker + s * workers, s);
    const float inv = 1.0f / (float)p.width;
    float sw[VALUES], sb[VALUES];
#pragma unroll
    for (int k = 0; k < VALUES; ++k) sw[k] = sb[k] = 0.0f;
    int place = 0, turn = 0;
    uint32_t parity = 0;
    bool there = true;                                       // a copy that did not come within the wait's limit: nothing is waited for any more
    for (int64_t t = worker; t < p.tokens; t += workers) {
        const float mu = p.mean != nullptr ? p.mean[t] : 0.0f, r = p.rstd[t];
        if (there) there = mbar_wait(smem_u32(&full[mine][place]), parity, &bars->abort_flag, q.timeout_word, TO_PRODUCER);
        const uint8_t* xs = ring + (size_t)place * 2 * q.row_bytes;
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int n = 0; n < VALUES / V; ++n) {
            const int c = (n * share + rank) * V;
            if (c >= p.width) break;
            float x[V], g[V], w[V];
            Elem<T>::unpack(*reinterpret_cast<const uint4*>(xs + c * sizeof(T)), x);
            Elem<T>::unpack(*reinterpret_cast<const uint4*>(xs + q.row_bytes + c * sizeof(T)), g);
            load_params<P, V>(reinterpret_cast<const P*>(p.weight), c, w);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xh = (x[e] - mu) * r;
                sw[n * V + e] = fmaf(g[e], xh, sw[n * V + e]);
                sb[n * V + e] += g[e];
                g[e] *= w[e];
                s[0] += g[e];
                s[1] = fmaf(g[e], xh, s[1]);
            }
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) { s[0] += __shfl_xor_sync(0xFFFFFFFFu, s[0], d); s[1] += __shfl_xor_sync(0xFFFFFFFFu, s[1], d); }
        if (warps > 1) {
            if (lane == 0) { room[mine][turn][warp_of][0] = s[0]; room[mine][turn][warp_of][1] = s[1]; }
            asm volatile("bar.sync %0, %1;" ::"r"(mine + 1), "r"(share) : "memory");
#pragma unroll
            for (int k = 0; k < 2; ++k) {                    // (in row_sum's order: dx is the same with and without the sums)
                s[k] = lane < warps ? room[mine][turn][lane][k] : 0.0f;
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) s[k] += __shfl_xor_sync(0xFFFFFFFFu, s[k], d);
            }
            turn ^= 1;
        } else {
            __syncwarp();
        }
        // every thread of the worker has left the row before: its place takes the row that is `stages` behind it
        if (rank == 0 && t > worker) {
            const int64_t next = t + (int64_t)(q.stages - 1) * workers;
            if (next < p.tokens && there) bring(next, place == 0 ? q.stages - 1 : place - 1);
        }
        const float m = p.center ? s[0] * inv : 0.0f, along = s[1] * inv;
        T* out = reinterpret_cast<T*>(p.out) + t * p.ld_out;
#pragma unroll
        for (int n = 0; n < VALUES / V; ++n) {
            const int c = (n * share + rank) * V;
            if (c >= p.width) break;
            float x[V], g[V], w[V];
            Elem<T>::unpack(*reinterpret_cast<const uint4*>(xs + c * sizeof(T)), x);
            Elem<T>::unpack(*reinterpret_cast<const uint4*>(xs + q.row_bytes + c * sizeof(T)), g);
            load_params<P, V>(reinterpret_cast<const P*>(p.weight), c, w);
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = (__fmul_rn(g[e], w[e]) - m - __fmul_rn(x[e] - mu, r) * along) * r;
            store_vec<T, V>(out + c, x);
        }
        if (++place == q.stages) { place = 0; parity ^= 1u; }
    }
    float* dst = p.part + worker * 2 * p.width;
#pragma unroll
    for (int n = 0; n < VALUES / V; ++n) {
        const int c = (n * share + rank) * V;
        if (c >= p.width) break;
#pragma unroll
        for (int e = 0; e < V; e += 4) {
            *reinterpret_cast<float4*>(dst + c + e) = make_float4(sw[n * V + e], sw[n * V + e + 1], sw[n * V + e + 2], sw[n * V + e + 3]);
            *reinterpret_cast<float4*>(dst + p.width + c + e) = make_float4(sb[n * V + e], sb[n * V + e + 1], sb[n * V + e + 2], sb[n * V + e + 3]);
        }
    }
    // behind a wait that gave up: what is still on its way arrives before the block leaves
    if (!there && rank == 0)
        for (int s = 0; s < q.stages; ++s) mbar_wait_quiet(smem_u32(&full[mine][s]), 0u, 1u << 14);
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

NormPlan plan_norm(int64_t tokens, int32_t width, int32_t elem, bool sums)
{
    NormPlan pl;
    pl.share = width <= 32 * VALUES ? 32 : width <= 128 * VALUES ? 128 : width <= 256 * VALUES ? 256 : 512;
    pl.block = pl.share > ROOM_BLOCK ? pl.share : ROOM_BLOCK;
    if (pl.share == 128 && !sums) pl.block = 128;            // (the barriers of the plain kernels are a block's)
    const int64_t per = pl.block / pl.share, all = (tokens + per - 1) / per, sms = sm_count();
    pl.blocks = all;
    pl.workers = pl.ring_workers = all * per;
    pl.ring_stages = 0;
    pl.total = 256;
    if (!sums) return pl;
    // Two blocks an SM with some 96 KiB of rows on their way each.
    const int64_t stages = (96 << 10) / (per * 2 * width * (int64_t)elem);
    pl.ring_stages = (int32_t)(stages > 8 ? 8 : stages);
    pl.ring_workers = (all < 2 * sms ? all : 2 * sms) * per;
    // without the ring: as many blocks as are resident
    if (pl.share == 128) { pl.block = 128; pl.blocks = tokens; }
    const int64_t most = sms * (pl.block == 128 ? 3 : 1);
    if (pl.blocks > most) pl.blocks = most;
    pl.workers = pl.blocks * (pl.block / pl.share);
    const int64_t rows = pl.workers > pl.ring_workers ? pl.workers : pl.ring_workers;
    pl.total = align_up((size_t)rows * 2 * width * 4, 256) + 256;
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
    const int es = a.dtype == QLESS_F32 ? 4 : 2, vec = 16 / es;
    const NormPlan pl = plan_norm(a.tokens, a.width, es, false);
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

template <typename T, typename P>
static cudaError_t ring_of(const NormPlan& pl, const RingParams& q, cudaStream_t st)
{
    const cudaError_t e = allow_full_smem<norm_backward_ring_kernel<T, P>>();
    if (e != cudaSuccess) return e;
    const size_t smem = sizeof(RingBars) + (size_t)(256 / pl.share) * pl.ring_stages * 2 * q.row_bytes;
    return launch_ahead(norm_backward_ring_kernel<T, P>, dim3((unsigned)(pl.ring_workers / (256 / pl.share))), dim3(256), smem, st, q);
}

qless_status launch_norm_backward(const NormArgs& a, uint8_t* ws, unsigned int* timeout_word, cudaStream_t st)
{
    const bool sums = a.grad_weight != nullptr || a.grad_bias != nullptr;
    const int es = a.dtype == QLESS_F32 ? 4 : 2, vec = 16 / es;
    const NormPlan pl = plan_norm(a.tokens, a.width, es, sums);
    const bool whole = a.width % vec == 0 && vectors(a.x, a.ld_x, es) && vectors(a.dy, a.ld_dy, es) && vectors(a.out, a.ld_out, es) && vectors(a.weight, 0, 1);
    NormParams p{};
    p.x = a.x; p.dy = a.dy; p.weight = a.weight; p.out = a.out; p.mean = a.center ? a.mean : nullptr; p.rstd = a.rstd; p.part = reinterpret_cast<float*>(ws);
    p.tokens = a.tokens; p.ld_x = a.ld_x; p.ld_dy = a.ld_dy; p.ld_out = a.ld_out; p.width = a.width; p.share = pl.share; p.center = a.center;
    const bool ring = sums && whole && pl.share <= 256 && pl.ring_stages >= 2;
    const int64_t workers = ring ? pl.ring_workers : pl.workers;
    { ProfileScope ps("layer_norm_backward", st);
      if (ring) {
          RingParams q{};
          q.n = p; q.stages = pl.ring_stages; q.row_bytes = a.width * es; q.timeout_word = timeout_word;
          if (a.dtype == QLESS_F32) {
              if (a.param_dtype == QLESS_F32) QLESS_CUDA_TRY((ring_of<float, float>(pl, q, st)));
              else QLESS_CUDA_TRY((ring_of<float, __nv_bfloat16>(pl, q, st)));
          } else {
              if (a.param_dtype == QLESS_F32) QLESS_CUDA_TRY((ring_of<__nv_bfloat16, float>(pl, q, st)));
              else QLESS_CUDA_TRY((ring_of<__nv_bfloat16, __nv_bfloat16>(pl, q, st)));
          }
      } else if (a.dtype == QLESS_F32) {
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
            QLESS_CUDA_TRY(launch_ahead(norm_join_kernel<float>, grid, dim3(1024), 0, st, part, workers, a.width, reinterpret_cast<float*>(a.grad_weight),
                                        reinterpret_cast<float*>(a.grad_bias)));
        else
            QLESS_CUDA_TRY(launch_ahead(norm_join_kernel<__nv_bfloat16>, grid, dim3(1024), 0, st, part, workers, a.width,
                                        reinterpret_cast<__nv_bfloat16*>(a.grad_weight), reinterpret_cast<__nv_bfloat16*>(a.grad_bias)));
        count_launches(1);
    }
    return QLESS_OK;
}

}  // namespace qless
