// Layer normalisation of the rows of a matrix, forward and backward (with `center` off: by the root mean square alone).
//
//   mu = mean x (0 without centring),  r = 1 / sqrt(mean (x - mu)^2 + eps),  xh = (x - mu) r,  y = xh w + b
//   g = w dy;  dx = r (g - mean g - xh mean(g xh)) (no mean g without centring);  dw = sum_t dy xh;  db = sum_t dy
//
// Bound: bytes (forward: x read, y written; backward: x and dy read, dx written; a few operations an element). A row is read once: its
// values stay in the registers of the threads that share it (four 16-byte vectors a thread where rows are aligned, else 16 values, element by
// element with neighbouring lanes on neighbouring elements), and the moments are taken from them in two steps, mean and then squares
// of the differences: squares lose nothing to a mean far from zero (the mean itself is an fp32 sum, off by some 2^-23 of the values' size, and so are the differences). The fewest warps that hold a row share it.
// dw and db: workers that walk over the rows keep their columns' sums in registers and leave one row of fp32 sums each, which a second
// kernel adds in a fixed order (no atomics: the same inputs give the same bits). With the sums there is no room to hold rows ahead in
// registers, and few warps an SM: aligned rows of up to 32 KiB come through a ring in shared memory (norm_backward_ring_kernel). Its arithmetic works on pairs
// of values. With the copies ahead neither bytes (DRAM 45 % busy at 4112 columns) nor instructions (49 % of the issue slots) bound it: a worker's two passes over a row and the
// barrier between them follow one another. 65521 x 4112 bf16: 370 us with the parameters' gradients, 400 without (no ring there).
#include "pairs.cuh"
#include "qless_kernels.h"
#include "tc_common.cuh"

namespace qless {

namespace {

// Values of a row that one thread holds.
__host__ __device__ constexpr int values_of(int V) { return V == 1 ? 16 : 4 * V; }

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

// A thread's values of a row come in slots, of a vector each or (V = 1) of two single elements `share` apart: element e of slot n.
template <int V> constexpr int SLOT = V == 1 ? 2 : V;
template <int V> constexpr int SLOTS = values_of(V) / SLOT<V>;
template <int V> __device__ __forceinline__ int column(int n, int e, int rank, int share) { return V == 1 ? (2 * n + e) * share + rank : (n * share + rank) * V + e; }

template <typename T, int V>
__device__ __forceinline__ void load_slot(const T* row, int n, int width, int rank, int share, float* v)      // zeros behind the row
{
    const int c = column<V>(n, 0, rank, share);
    if constexpr (V == 1) {
        v[0] = c < width ? Elem<T>::get(row + c) : 0.0f;
        v[1] = c + share < width ? Elem<T>::get(row + c + share) : 0.0f;
    } else {
        uint4 u = make_uint4(0u, 0u, 0u, 0u);
        if (c < width) u = __ldg(reinterpret_cast<const uint4*>(row + c));
        Elem<T>::unpack(u, v);
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_slot(T* row, int n, int width, int rank, int share, const float* v)
{
    const int c = column<V>(n, 0, rank, share);
    if constexpr (V == 1) {
        if (c < width) Elem<T>::put(row + c, v[0]);
        if (c + share < width) Elem<T>::put(row + c + share, v[1]);
    } else if (c < width) {
        *reinterpret_cast<uint4*>(row + c) = Elem<T>::pack(v);
    }
}
// The parameters of a slot, whatever their type (zeros behind the row).
template <typename P, int V>
__device__ __forceinline__ void load_params(const P* p, int n, int width, int rank, int share, float* v)
{
    const int c = column<V>(n, 0, rank, share);
    if constexpr (V == 1) {
        v[0] = c < width ? Elem<P>::get(p + c) : 0.0f;
        v[1] = c + share < width ? Elem<P>::get(p + c + share) : 0.0f;
    } else if (c >= width) {
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = 0.0f;
    } else if constexpr (Elem<P>::VEC <= V) {
#pragma unroll
        for (int k = 0; k < V; k += Elem<P>::VEC) Elem<P>::unpack(__ldg(reinterpret_cast<const uint4*>(p + c + k)), v + k);
    } else {                                                 // four bf16 parameters beside four fp32 values
        const uint2 u = __ldg(reinterpret_cast<const uint2*>(p + c));
        v[0] = __uint_as_float(u.x << 16); v[1] = __uint_as_float(u.x & 0xFFFF0000u);
        v[2] = __uint_as_float(u.y << 16); v[3] = __uint_as_float(u.y & 0xFFFF0000u);
    }
}

// Sums of K numbers over the threads that share a row (a warp, or the whole block), in every one of them. `room` alternates between two halves,
// so that one barrier per call is enough: a half is written again only behind the barrier of the call after.
template <int K>
__device__ __forceinline__ void row_sum(float (&x)[K], int share, float (*room)[32][2], int& turn)
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
    const int warps = share >> 5, half = 1 << (31 - __clz(warps - 1)), at = lane & (2 * half - 1);      // half: of the next power of two
#pragma unroll
    for (int k = 0; k < K; ++k) {
        x[k] = at < warps ? room[turn][at][k] : 0.0f;
        for (int s = half; s > 0; s >>= 1) x[k] += __shfl_xor_sync(0xFFFFFFFFu, x[k], s);
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

template <typename T, typename P, int V, int BLOCK>
__global__ void __launch_bounds__(BLOCK) norm_forward_kernel(const NormParams p)
{
    __shared__ float room[2][32][2];
    ahead_wait();
    ahead_release();
    int turn = 0;
    const int share = p.share, rank = threadIdx.x % share;
    const int64_t t = (int64_t)blockIdx.x * (blockDim.x / share) + threadIdx.x / share;
    if (t >= p.tokens) return;                               // whole warps: a block of one row has it
    constexpr int S = SLOT<V>, N = SLOTS<V>;
    float v[N * S];
#pragma unroll
    for (int n = 0; n < N; ++n) load_slot<T, V>(reinterpret_cast<const T*>(p.x) + t * p.ld_x, n, p.width, rank, share, v + n * S);
    const float inv = 1.0f / (float)p.width;
    float mu = 0.0f;
    if (p.center) {
        float s[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < N * S; ++k) s[0] += v[k];        // places behind the row hold 0
        row_sum<1>(s, share, room, turn);
        mu = s[0] * inv;
    }
    float s[1] = {0.0f};
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (column<V>(n, 0, rank, share) >= p.width) break;
#pragma unroll
        for (int e = 0; e < S; ++e) {
            float& x = v[n * S + e];
            x -= mu;
            if (V == 1 && e == 1 && column<V>(n, 1, rank, share) >= p.width) x = 0.0f;
            s[0] = fmaf(x, x, s[0]);
        }
    }
    row_sum<1>(s, share, room, turn);
    const float r = rsqrtf(fmaf(s[0], inv, p.eps));
    if (rank == 0) {
        if (p.mean != nullptr) p.mean[t] = mu;
        if (p.rstd != nullptr) p.rstd[t] = r;
    }
    T* out = reinterpret_cast<T*>(p.out) + t * p.ld_out;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (column<V>(n, 0, rank, share) >= p.width) break;
        float w[S], b[S], y[S];
        load_params<P, V>(reinterpret_cast<const P*>(p.weight), n, p.width, rank, share, w);
        if (p.bias != nullptr) load_params<P, V>(reinterpret_cast<const P*>(p.bias), n, p.width, rank, share, b);
#pragma unroll
        for (int e = 0; e < S; ++e) y[e] = p.bias != nullptr ? fmaf(v[n * S + e] * r, w[e], b[e]) : v[n * S + e] * r * w[e];
        store_slot<T, V>(out, n, p.width, rank, share, y);
    }
}

// A row's backward pass in three steps, the same in both kernels, so that dx has the same bits with and without the sums. With d = x - mu, g = w dy:
//   (1) sums of g and of g d (and, by column, of dy and r dy d)   (2) over the threads   (3) dx = (d r) A + (g r - m r),  m = mean g,  A = -r (mean(g d) r)
// (d r is formed first and the factors of A in this order because r^2 and r^3 leave fp32's range where r and dx do not: a spread of 5e-20 or less, with eps = 0.)
struct RowSums { uint64_t g = 0, gd = 0; };

template <int S, bool SUMS>
__device__ __forceinline__ void add_slot(const float* x, const float* dy, const float* w, float mu, float r, RowSums& sums, uint64_t* sw, uint64_t* sb)
{
    const uint64_t mu2 = pair_of(-mu, -mu), r2 = pair_of(r, r);
#pragma unroll
    for (int k = 0; k < S / 2; ++k) {
        const uint64_t dy2 = pair_of(dy[2 * k], dy[2 * k + 1]), d = add2(pair_of(x[2 * k], x[2 * k + 1]), mu2);
        if (SUMS) { sw[k] = fma2(mul2(dy2, r2), d, sw[k]); sb[k] = add2(sb[k], dy2); }
        const uint64_t g = mul2(dy2, pair_of(w[2 * k], w[2 * k + 1]));
        sums.g = add2(sums.g, g);
        sums.gd = fma2(g, d, sums.gd);
    }
}
__device__ __forceinline__ void close_sums(const RowSums& sums, float (&s)[2])
{
    float a, b;
    split_pair(sums.g, a, b);
    s[0] = a + b;
    split_pair(sums.gd, a, b);
    s[1] = a + b;
}
template <int S>
__device__ __forceinline__ void form_slot(const float* x, const float* dy, const float* w, float mu, float r, float by_xh, float shift, float* dx)
{
    const uint64_t mu2 = pair_of(-mu, -mu), r2 = pair_of(r, r), a2 = pair_of(by_xh, by_xh), s2 = pair_of(shift, shift);
#pragma unroll
    for (int k = 0; k < S / 2; ++k) {
        const uint64_t g = mul2(pair_of(dy[2 * k], dy[2 * k + 1]), pair_of(w[2 * k], w[2 * k + 1])), d = add2(pair_of(x[2 * k], x[2 * k + 1]), mu2);
        split_pair(fma2(mul2(d, r2), a2, fma2(g, r2, s2)), dx[2 * k], dx[2 * k + 1]);
    }
}

// A worker (the threads that share a row) takes every workers-th row; SUMS: it keeps its columns' sums and leaves them in part.
template <typename T, typename P, int V, bool SUMS, int BLOCK>
__global__ void __launch_bounds__(BLOCK) norm_backward_kernel(const NormParams p)
{
    __shared__ float room[2][32][2];
    ahead_wait();
    ahead_release();
    int turn = 0;
    const int share = p.share, rank = threadIdx.x % share, per = blockDim.x / share;
    const int64_t worker = (int64_t)blockIdx.x * per + threadIdx.x / share, workers = (int64_t)gridDim.x * per;
    const float inv = 1.0f / (float)p.width;
    constexpr int S = SLOT<V>, N = SLOTS<V>;
    uint64_t sw[SUMS ? N * S / 2 : 1], sb[SUMS ? N * S / 2 : 1];
    if (SUMS) {
#pragma unroll
        for (int k = 0; k < N * S / 2; ++k) sw[k] = sb[k] = 0;
    }
    for (int64_t t = worker; t < p.tokens; t += workers) {   // (a block of one worker: the same trips for all of its threads)
        float x[N * S], dy[N * S];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            load_slot<T, V>(reinterpret_cast<const T*>(p.x) + t * p.ld_x, n, p.width, rank, share, x + n * S);
            load_slot<T, V>(reinterpret_cast<const T*>(p.dy) + t * p.ld_dy, n, p.width, rank, share, dy + n * S);
        }
        const float mu = p.mean != nullptr ? p.mean[t] : 0.0f, r = p.rstd[t];
        RowSums sums;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (column<V>(n, 0, rank, share) >= p.width) break;
            float w[S];
            load_params<P, V>(reinterpret_cast<const P*>(p.weight), n, p.width, rank, share, w);
            add_slot<S, SUMS>(x + n * S, dy + n * S, w, mu, r, sums, sw + (SUMS ? n * S / 2 : 0), sb + (SUMS ? n * S / 2 : 0));
        }
        float s[2];
        close_sums(sums, s);
        row_sum<2>(s, share, room, turn);
        const float by_xh = -r * (s[1] * inv * r), shift = p.center ? -s[0] * inv * r : 0.0f;
        T* out = reinterpret_cast<T*>(p.out) + t * p.ld_out;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (column<V>(n, 0, rank, share) >= p.width) break;
            float w[S], dx[S];
            load_params<P, V>(reinterpret_cast<const P*>(p.weight), n, p.width, rank, share, w);
            form_slot<S>(x + n * S, dy + n * S, w, mu, r, by_xh, shift, dx);
            store_slot<T, V>(out, n, p.width, rank, share, dx);
        }
    }
    if (SUMS) {
        float* dst = p.part + worker * 2 * p.width;
#pragma unroll
        for (int k = 0; k < N * S / 2; ++k) {
            float a[2], b[2];
            split_pair(sw[k], a[0], a[1]);
            split_pair(sb[k], b[0], b[1]);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int c = column<V>(2 * k / S, 2 * k % S + e, rank, share);
                if (c < p.width) { dst[c] = a[e]; dst[p.width + c] = b[e]; }
            }
        }
    }
}

// The same with the sums, rows brought ahead by bulk copies: every worker has a ring of `stages` places of a row of x and one of dy. EIGHTS: columns
// of a thread, in eights. A row is read from its place twice (for the two means, then for dx); the place is filled again behind the barrier of the next
// row's means, when every thread of the worker has left it. (Two rows at a time, which share a barrier and the weights' unpacking: 32768 rows of
// 2048 bf16 96 us, 4096 fp32 287; one at a time 95 and 273. 65521 x 4112 bf16: 368 us.)
struct RingParams {
    NormParams n;
    int32_t stages, row_bytes;
    unsigned int* timeout_word;
};

struct __align__(128) RingBars {
    uint64_t full[8][8];                    // [worker of the block][place]
    float room[2][16][2];                   // [turn][warp][means of a row], of a worker of several warps
    uint32_t abort_flag;
};

template <typename T, typename P, int EIGHTS>
__global__ void __launch_bounds__(512, 1) norm_backward_ring_kernel(const RingParams q)
{
    using namespace tc;
    constexpr int V = Elem<T>::VEC, N = EIGHTS * 8 / V;
    extern __shared__ __align__(128) uint8_t smem[];
    RingBars* bars = reinterpret_cast<RingBars*>(smem);
    const NormParams& p = q.n;
    const int share = p.share, rank = threadIdx.x % share, mine = threadIdx.x / share, per = blockDim.x / share;
    const int lane = threadIdx.x & 31, warp_of = rank >> 5, warps = share >> 5;
    const int half = warps > 1 ? 1 << (31 - __clz(warps - 1)) : 0, at = lane & (2 * half - 1);      // (as in row_sum)
    uint64_t* full = bars->full[mine];
    float (*room)[16][2] = bars->room;
    if (threadIdx.x == 0) {
        for (int i = 0; i < per; ++i) for (int s = 0; s < q.stages; ++s) mbar_init(smem_u32(&bars->full[i][s]), 1);
        bars->abort_flag = 0;
        fence_barrier_init();
    }
    __syncthreads();
    ahead_wait();
    ahead_release();
    const int64_t worker = (int64_t)blockIdx.x * per + mine, workers = (int64_t)gridDim.x * per;
    uint8_t* ring = smem + sizeof(RingBars) + (size_t)mine * q.stages * 2 * q.row_bytes;
    auto bring = [&](int64_t t, int place) {                 // one thread
        const uint32_t bar = smem_u32(&full[place]), dst = smem_u32(ring + (size_t)place * 2 * q.row_bytes);
        mbar_arrive_expect_tx(bar, 2 * q.row_bytes);
        bulk_load(dst, reinterpret_cast<const T*>(p.x) + t * p.ld_x, q.row_bytes, bar);
        bulk_load(dst + q.row_bytes, reinterpret_cast<const T*>(p.dy) + t * p.ld_dy, q.row_bytes, bar);
    };
    if (rank == 0)
        for (int s = 0; s < q.stages && worker + s * workers < p.tokens; ++s) bring(worker + s * workers, s);
    const float inv = 1.0f / (float)p.width;
    uint64_t sw[N * V / 2], sb[N * V / 2];
#pragma unroll
    for (int k = 0; k < N * V / 2; ++k) sw[k] = sb[k] = 0;
    int place = 0, turn = 0;
    uint32_t parity = 0;
    float mu_next = 0.0f, r_next = 0.0f;
    bool there = true;                                       // a copy that did not come within the wait's limit: nothing is waited for any more
    auto stats = [&](int64_t t) {
        if (t < p.tokens) {
            mu_next = p.mean != nullptr ? p.mean[t] : 0.0f;
            r_next = p.rstd[t];
        }
    };
    stats(worker);
    for (int64_t t = worker; t < p.tokens; t += workers) {
        const float mu = mu_next, r = r_next;
        stats(t + workers);
        if (there) there = mbar_wait(smem_u32(&full[place]), parity, &bars->abort_flag, q.timeout_word, TO_PRODUCER);
        const uint8_t* xs = ring + (size_t)place * 2 * q.row_bytes;
        auto values = [&](int c, float* x, float* dy) {
            Elem<T>::unpack(*reinterpret_cast<const uint4*>(xs + c * sizeof(T)), x);
            Elem<T>::unpack(*reinterpret_cast<const uint4*>(xs + q.row_bytes + c * sizeof(T)), dy);
        };
        RowSums sums;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = column<V>(n, 0, rank, share);
            if (c >= p.width) break;
            float w[V], x[V], dy[V];
            load_params<P, V>(reinterpret_cast<const P*>(p.weight), n, p.width, rank, share, w);
            values(c, x, dy);
            add_slot<V, true>(x, dy, w, mu, r, sums, sw + n * V / 2, sb + n * V / 2);
        }
        float s[2];
        close_sums(sums, s);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            s[0] += __shfl_xor_sync(0xFFFFFFFFu, s[0], d);
            s[1] += __shfl_xor_sync(0xFFFFFFFFu, s[1], d);
        }
        if (warps > 1) {                                     // (in row_sum's order)
            if (lane == 0) { room[turn][warp_of][0] = s[0]; room[turn][warp_of][1] = s[1]; }
            __syncthreads();                                 // (the block is this worker)
            s[0] = at < warps ? room[turn][at][0] : 0.0f;
            s[1] = at < warps ? room[turn][at][1] : 0.0f;
            for (int d = half; d > 0; d >>= 1) {
                s[0] += __shfl_xor_sync(0xFFFFFFFFu, s[0], d);
                s[1] += __shfl_xor_sync(0xFFFFFFFFu, s[1], d);
            }
            turn ^= 1;
        } else {
            __syncwarp();
        }
        // every thread of the worker has left the row before: its place takes the row that is `stages` behind it
        if (rank == 0 && t > worker && there) {
            const int64_t next = t + (int64_t)(q.stages - 1) * workers;
            if (next < p.tokens) bring(next, place >= 1 ? place - 1 : q.stages - 1);
        }
        const float by_xh = -r * (s[1] * inv * r), shift = p.center ? -s[0] * inv * r : 0.0f;
        T* out = reinterpret_cast<T*>(p.out) + t * p.ld_out;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = column<V>(n, 0, rank, share);
            if (c >= p.width) break;
            float w[V], x[V], dy[V], dx[V];
            load_params<P, V>(reinterpret_cast<const P*>(p.weight), n, p.width, rank, share, w);
            values(c, x, dy);
            form_slot<V>(x, dy, w, mu, r, by_xh, shift, dx);
            store_slot<T, V>(out, n, p.width, rank, share, dx);
        }
        if (++place == q.stages) { place = 0; parity ^= 1u; }
    }
    float* dst = p.part + worker * 2 * p.width;
#pragma unroll
    for (int k = 0; k < N * V / 2; k += 2) {
        const int c = column<V>(2 * k / V, 2 * k % V, rank, share);
        if (c >= p.width) break;
        float a[4], b[4];
        split_pair(sw[k], a[0], a[1]);
        split_pair(sw[k + 1], a[2], a[3]);
        split_pair(sb[k], b[0], b[1]);
        split_pair(sb[k + 1], b[2], b[3]);
        *reinterpret_cast<float4*>(dst + c) = make_float4(a[0], a[1], a[2], a[3]);
        *reinterpret_cast<float4*>(dst + p.width + c) = make_float4(b[0], b[1], b[2], b[3]);
    }
    // behind a wait that gave up: what is still on its way arrives before the block leaves
    if (!there && rank == 0)
        for (int s = 0; s < q.stages; ++s) mbar_wait_quiet(smem_u32(&full[s]), parity ^ (s < place ? 1u : 0u), 1u << 14);
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
    if (c < width) {
#pragma unroll 4
        for (int64_t k = warp; k < workers; k += 32) s += part[(2 * k + which) * width + c];
    }
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

struct NormPlan { int32_t share, block, ring_stages; int64_t blocks, workers; size_t total; };

// elem: bytes of a value; whole: rows of whole vectors.
NormPlan plan_norm(int64_t tokens, int32_t width, int32_t elem, bool sums, bool whole)
{
    NormPlan pl;
    const int32_t values = values_of(whole ? 16 / elem : 1);
    pl.share = (width + 32 * values - 1) / (32 * values) * 32;
    pl.block = pl.share > 32 ? pl.share : 256;               // several rows to a block only where a warp has one
    const int64_t per = pl.block / pl.share, sms = sm_count();
    pl.blocks = (tokens + per - 1) / per;
    const bool ring = sums && whole && pl.share <= 512 && (int64_t)width * elem <= 32768;
    int64_t resident = pl.block <= 512 ? 65536 / (128 * pl.block) : 1;      // blocks an SM, with 128 registers a thread
    pl.ring_stages = 0;
    if (ring) {
        // Some 200 KiB of rows on their way an SM, at least three to a worker.
        const int64_t row = per * 2 * width * (int64_t)elem, room = 200 << 10;
        while (resident > 1 && room / resident < 3 * row) --resident;
        const int64_t stages = room / resident / row;
        pl.ring_stages = (int32_t)(stages > 8 ? 8 : stages);
    }
    // Workers that keep sums: as many as are resident.
    const int64_t most = sms * resident;
    if (sums && pl.blocks > most) pl.blocks = most;
    pl.workers = pl.blocks * per;
    pl.total = sums ? align_up((size_t)pl.workers * 2 * width * 4, 256) + 256 : 256;
    return pl;
}

template <typename T, typename P, int V>
cudaError_t forward_of(const NormPlan& pl, const NormParams& p, cudaStream_t st)
{
    const dim3 grid((unsigned)pl.blocks), block((unsigned)pl.block);
    return pl.block <= 256 ? launch_ahead(norm_forward_kernel<T, P, V, 256>, grid, block, 0, st, p) : launch_ahead(norm_forward_kernel<T, P, V, 1024>, grid, block, 0, st, p);
}

template <typename T, typename P, int V, bool SUMS>
cudaError_t backward_of(const NormPlan& pl, const NormParams& p, cudaStream_t st)
{
    const dim3 grid((unsigned)pl.blocks), block((unsigned)pl.block);
    if (pl.block <= 256) return launch_ahead(norm_backward_kernel<T, P, V, SUMS, 256>, grid, block, 0, st, p);
    if constexpr (V < 8)                                     // (vectors of bf16: 16384 values are 512 threads')
        if (pl.block > 512) return launch_ahead(norm_backward_kernel<T, P, V, SUMS, 1024>, grid, block, 0, st, p);
    return launch_ahead(norm_backward_kernel<T, P, V, SUMS, 512>, grid, block, 0, st, p);
}

// With the sums and without a ring: rows that are not whole vectors, and fp32 rows beyond 32 KiB, which have more than 512 threads. (Whole bf16 rows always take the ring.)
template <typename T, typename P>
cudaError_t sums_of(const NormPlan& pl, const NormParams& p, bool whole, cudaStream_t st)
{
    if constexpr (sizeof(T) == 4)
        if (whole) return launch_ahead(norm_backward_kernel<T, P, 4, true, 1024>, dim3((unsigned)pl.blocks), dim3((unsigned)pl.block), 0, st, p);
    return backward_of<T, P, 1, true>(pl, p, st);
}

template <typename T, typename P, int EIGHTS>
cudaError_t ring_as(const NormPlan& pl, const RingParams& q, cudaStream_t st)
{
    const cudaError_t e = allow_full_smem<norm_backward_ring_kernel<T, P, EIGHTS>>();
    if (e != cudaSuccess) return e;
    const size_t smem = sizeof(RingBars) + (size_t)(pl.block / pl.share) * pl.ring_stages * 2 * q.row_bytes;
    return launch_ahead(norm_backward_ring_kernel<T, P, EIGHTS>, dim3((unsigned)pl.blocks), dim3((unsigned)pl.block), smem, st, q);
}

template <typename T, typename P>
cudaError_t ring_of(const NormPlan& pl, const RingParams& q, cudaStream_t st)
{
    const int eights = (q.n.width + 8 * pl.share - 1) / (8 * pl.share);
    if (eights == 1) return ring_as<T, P, 1>(pl, q, st);
    if constexpr (sizeof(T) == 4) {
        return ring_as<T, P, 2>(pl, q, st);
    } else {
        if (eights == 2) return ring_as<T, P, 2>(pl, q, st);
        if (eights == 3) return ring_as<T, P, 3>(pl, q, st);
        return ring_as<T, P, 4>(pl, q, st);
    }
}

// Whole vectors: the rows' width, their addresses and the parameters' allow 16-byte accesses.
bool whole_rows(const NormArgs& a, int es)
{
    return a.width % (16 / es) == 0 && vectors(a.x, a.ld_x, es) && vectors(a.out, a.ld_out, es) && (a.dy == nullptr || vectors(a.dy, a.ld_dy, es)) &&
           vectors(a.weight, 0, 1) && (a.bias == nullptr || vectors(a.bias, 0, 1));
}

}  // namespace

size_t norm_workspace(const NormArgs& a)
{
    const int es = a.dtype == QLESS_F32 ? 4 : 2;
    return plan_norm(a.tokens, a.width, es, a.grad_weight != nullptr || a.grad_bias != nullptr, whole_rows(a, es)).total;
}

size_t norm_most_workspace(int64_t tokens, int32_t width, bool sums)
{
    size_t most = 256;
    for (int k = 0; k < 4; ++k) {
        const size_t one = plan_norm(tokens, width, k & 1 ? 4 : 2, sums, (k & 2) != 0).total;
        if (one > most) most = one;
    }
    return most;
}

#define QLESS_BY_TYPES(CALL)                                                                       \
    do {                                                                                           \
        if (a.dtype == QLESS_F32) {                                                                \
            if (a.param_dtype == QLESS_F32) QLESS_CUDA_TRY((CALL(float, float)));                  \
            else QLESS_CUDA_TRY((CALL(float, __nv_bfloat16)));                                     \
        } else {                                                                                   \
            if (a.param_dtype == QLESS_F32) QLESS_CUDA_TRY((CALL(__nv_bfloat16, float)));          \
            else QLESS_CUDA_TRY((CALL(__nv_bfloat16, __nv_bfloat16)));                             \
        }                                                                                          \
    } while (0)

qless_status launch_norm_forward(const NormArgs& a, cudaStream_t st)
{
    const int es = a.dtype == QLESS_F32 ? 4 : 2;
    const bool whole = whole_rows(a, es);
    const NormPlan pl = plan_norm(a.tokens, a.width, es, false, whole);
    NormParams p{};
    p.x = a.x; p.weight = a.weight; p.bias = a.bias; p.out = a.out; p.mean = a.mean; p.rstd = a.rstd;
    p.tokens = a.tokens; p.ld_x = a.ld_x; p.ld_out = a.ld_out; p.width = a.width; p.share = pl.share; p.center = a.center; p.eps = a.eps;
    ProfileScope ps("layer_norm", st);
#define QLESS_CALL(T, P) whole ? forward_of<T, P, Elem<T>::VEC>(pl, p, st) : forward_of<T, P, 1>(pl, p, st)
    QLESS_BY_TYPES(QLESS_CALL);
#undef QLESS_CALL
    count_launches(1);
    return QLESS_OK;
}

qless_status launch_norm_backward(const NormArgs& a, uint8_t* ws, unsigned int* timeout_word, cudaStream_t st)
{
    const bool sums = a.grad_weight != nullptr || a.grad_bias != nullptr;
    const int es = a.dtype == QLESS_F32 ? 4 : 2;
    const bool whole = whole_rows(a, es);
    const NormPlan pl = plan_norm(a.tokens, a.width, es, sums, whole);
    NormParams p{};
    p.x = a.x; p.dy = a.dy; p.weight = a.weight; p.out = a.out; p.mean = a.center ? a.mean : nullptr; p.rstd = a.rstd; p.part = reinterpret_cast<float*>(ws);
    p.tokens = a.tokens; p.ld_x = a.ld_x; p.ld_dy = a.ld_dy; p.ld_out = a.ld_out; p.width = a.width; p.share = pl.share; p.center = a.center;
    { ProfileScope ps("layer_norm_backward", st);
      if (pl.ring_stages > 0) {
          RingParams q{};
          q.n = p; q.stages = pl.ring_stages; q.row_bytes = a.width * es; q.timeout_word = timeout_word;
#define QLESS_CALL(T, P) ring_of<T, P>(pl, q, st)
          QLESS_BY_TYPES(QLESS_CALL);
#undef QLESS_CALL
      } else if (sums) {
#define QLESS_CALL(T, P) sums_of<T, P>(pl, p, whole, st)
          QLESS_BY_TYPES(QLESS_CALL);
#undef QLESS_CALL
      } else {
#define QLESS_CALL(T, P) whole ? backward_of<T, P, Elem<T>::VEC, false>(pl, p, st) : backward_of<T, P, 1, false>(pl, p, st)
          QLESS_BY_TYPES(QLESS_CALL);
#undef QLESS_CALL
      } }
    count_launches(1);
    if (sums) {
        ProfileScope ps("layer_norm_join", st);
        const dim3 grid((unsigned)(2 * ((a.width + 31) / 32)));
        const float* part = p.part;
        const int64_t workers = pl.workers;
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
