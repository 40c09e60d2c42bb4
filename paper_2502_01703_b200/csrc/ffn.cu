// Gated feed-forward block, forward and backward:  g = x Wg^T,  u = x Wu^T,  h = act(g) u,  y = h Wd^T
//
//   dh = dy Wd;  dg = dh u act'(g),  du = dh act(g);  dx = dg Wg + du Wu;  dWg = dg^T x,  dWu = du^T x,  dWd = dy^T h
//
// All products run in one kernel (ffn_gemm_kernel, tcgen05 on CTA pairs, 256 x 256 tiles, bf16 operands, fp32 accumulators in tensor memory, two of them
// so that the epilogue of a tile overlaps the next tile's products):
//   GLU        x [Wg; Wu]^T   a tile's 256 columns are 128 of g (rows of Wg, which the first CTA of the pair brings) and the same 128 of u (Wu, the
//                             second): the epilogue has both and writes h (and g and u where the backward pass wants them)
//   GLU_BACK   dy Wd          epilogue: dg, du (and h again, where the weights are trained) from the fp32 dh and the kept g and u
//   OUT        h Wd^T, dg Wg + du Wu (one contraction over both halves), dy^T h, and dg^T x with du^T x (two sets of tiles in one launch)
// Operands are read as they lie in memory, along the contraction or across it; what a tile's box has behind a matrix's edge arrives as zeros.
// Roundings to bf16: g, u where they are kept, h, dg, du (operands of the next product), and the results; every sum is fp32.
// Bound: the tensor pipe, at the clock that the power cap leaves (1.5 to 1.6 GHz). 4095 tokens x 4096 x 11008: dg and du 306 us (its epilogue reads and writes five matrices), dx
// 537 us (1.38 PFLOP/s). Few tokens are left to ffn_few.cu, where the weights' bytes bound.
#include <algorithm>

#include "ffn_common.cuh"

namespace qless {

using namespace ffn;

namespace {

constexpr int NTHREADS = 320;               // warp 0 TMA, warp 1 MMA, warps 2-9 epilogue (two groups of four)
constexpr int STAGES = 3;
constexpr int KB = 128;                     // contraction per stage: 64 KiB of operands per CTA
constexpr int HALF = 32768;
constexpr int GROUP_M = 16;                 // row tiles that share a pass over the column tiles

enum { GLU = 0, GLU_BACK = 1, OUT = 2 };

struct GemmParams {
    int32_t rows, cols;                     // of the result (GLU: cols = inner width)
    int32_t kblocks, kswitch;               // blocks of the contraction; from kswitch on the second operands are read
    int32_t sets;                           // OUT: 2 = a second result from the second left operand
    int32_t act;
    const __nv_bfloat16* gate_in; const __nv_bfloat16* up_in;
    __nv_bfloat16* out; __nv_bfloat16* out2; __nv_bfloat16* out3;      // GLU: h, g, u; GLU_BACK: dg, du, h; OUT: the results
    int64_t ld_gate_in, ld_up_in, ld, ld2, ld3;
    unsigned int* timeout_word;
};

struct __align__(8) Bars {
    uint64_t full[STAGES], empty[STAGES], d_full[2], d_empty[2], drain;
    uint32_t tmem_base, abort_flag;
};

struct Ring {
    uint32_t slot = 0, parity = 0;
    __device__ __forceinline__ void next(uint32_t n) { if (++slot == n) { slot = 0; parity ^= 1u; } }
};

// A_MN, B_MN: the operand's rows in memory run across the contraction.
template <int MODE, bool A_MN, bool B_MN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(NTHREADS, 1)
ffn_gemm_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const __grid_constant__ CUtensorMap tm_a2,
                const __grid_constant__ CUtensorMap tm_b2, const GemmParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    Bars* bars = reinterpret_cast<Bars*>(smem + STAGES * 2 * HALF);
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int64_t pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(smem_u32(&bars->full[s]), 1); mbar_init(smem_u32(&bars->empty[s]), 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&bars->d_full[s]), 1); mbar_init(smem_u32(&bars->d_empty[s]), 16); }
        mbar_init(smem_u32(&bars->drain), 1);
        bars->abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tm_a); prefetch_tmap(&tm_b); prefetch_tmap(&tm_a2); prefetch_tmap(&tm_b2);
    }
    if (warp == 1) { tmem_alloc_pair(smem_u32(&bars->tmem_base), 512); tmem_relinquish_pair(); }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;                   // accumulators at columns 0 and 256

    constexpr int TILE_N = MODE == GLU ? 128 : 256;          // columns of the result to a tile
    const int mt = (p.rows + 255) / 256, nt = (p.cols + TILE_N - 1) / TILE_N;
    const int64_t per_set = (int64_t)mt * nt, items = per_set * p.sets;
    // item -> (result, column tile, row tile): GROUP_M row tiles at a time, row tiles fastest
    auto item_of = [&](int64_t item, int& set, int& m, int& n) {
        set = item >= per_set ? 1 : 0;
        const int64_t r = item - set * per_set;
        const int64_t g = r / ((int64_t)GROUP_M * nt);
        const int m0 = (int)g * GROUP_M, gm = min(GROUP_M, mt - m0);
        const int rest = (int)(r - g * GROUP_M * nt);
        n = rest / gm;
        m = m0 + rest - n * gm;
    };
    auto warp_wait = [&](uint64_t* bar, uint32_t parity, uint32_t code) -> bool {
        const bool w = mbar_wait_cluster(smem_u32(bar), parity, abort_flag, p.timeout_word, code);
        return __all_sync(0xFFFFFFFFu, w);
    };

    if (warp == 0) {
        uint32_t it = 0;
        Ring ring;
        bool ok = true;
        for (int64_t item = pair; item < items && ok; item += num_pairs) {
            int set, m, n;
            item_of(item, set, m, n);
            const int a0 = m * 256 + (int)rank * 128, b0 = MODE == GLU ? n * 128 : n * 256 + (int)rank * 128;
            for (int kb = 0; kb < p.kblocks; ++kb, ++it, ring.next(STAGES)) {
                if (!warp_wait(&bars->empty[ring.slot], ring.parity ^ 1u, TO_PRODUCER)) { ok = false; break; }
                const uint32_t full = map_to_cta(smem_u32(&bars->full[ring.slot]), 0);
                const uint32_t a = smem_u32(smem + (size_t)ring.slot * 2 * HALF), b = a + HALF;
                const bool second = kb >= p.kswitch;
                const CUtensorMap* ma = second || set ? &tm_a2 : &tm_a;
                const CUtensorMap* mb = second || (MODE == GLU && rank != 0) ? &tm_b2 : &tm_b;
                const int k0 = (second ? kb - p.kswitch : kb) * KB;
                if (elect_one()) {
                    if (rank == 0) mbar_arrive_expect_tx(smem_u32(&bars->full[ring.slot]), 4 * HALF);      // both CTAs' bytes
                    for (int j = 0; j < 2; ++j) tma_load_2d_pair(a + j * 16384, ma, full, (A_MN ? a0 : k0) + 64 * j, A_MN ? k0 : a0);
                    for (int j = 0; j < 2; ++j) tma_load_2d_pair(b + j * 16384, mb, full, (B_MN ? b0 : k0) + 64 * j, B_MN ? k0 : b0);
                }
                __syncwarp();
            }
        }
        if (ok) ok = __all_sync(0xFFFFFFFFu, ring_drained(bars->empty, ring, STAGES, abort_flag, p.timeout_word, TO_PRODUCER));
        if (!ok) {           // leave no copy in flight: the leader waits (bounded) for the stages that are armed, the peer idles
            if (rank == 0) {
                for (uint32_t j = (it > STAGES ? it - STAGES : 0u); j < it; ++j)
                    if (!mbar_wait_quiet(smem_u32(&bars->full[j % STAGES]), (j / STAGES) & 1u, 1u << 14)) break;
            } else {
                for (uint32_t t = 0; t < (1u << 14); ++t) __nanosleep(64);
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            constexpr uint32_t idesc = make_idesc(1, 1, 1, 256, 256) | (A_MN ? IDESC_A_MN : 0u) | (B_MN ? IDESC_B_MN : 0u);
            Ring ring;
            uint32_t n_acc = 0;
            bool ok = true;
            for (int64_t item = pair; item < items && ok; item += num_pairs, ++n_acc) {
                const uint32_t buf = n_acc & 1u, d = tmem + buf * 256;
                if (!warp_wait(&bars->d_empty[buf], ((n_acc >> 1) & 1u) ^ 1u, TO_MMA)) { ok = false; break; }
                tc_fence_after();
                for (int kb = 0; kb < p.kblocks; ++kb, ring.next(STAGES)) {
                    // (an own barrier that only copies arrive on: no cluster-scope acquire)
                    bool landed = mbar_wait(smem_u32(&bars->full[ring.slot]), ring.parity, abort_flag, p.timeout_word, TO_MMA);
                    landed = __all_sync(0xFFFFFFFFu, landed);
                    if (!landed) { ok = false; break; }
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t a = smem_u32(smem + (size_t)ring.slot * 2 * HALF), b = a + HALF;
                        const uint64_t a0 = A_MN ? make_smem_desc_mn_sw128(a, 16384) : make_smem_desc_sw128(a);
                        const uint64_t b0 = B_MN ? make_smem_desc_mn_sw128(b, 16384) : make_smem_desc_sw128(b);
                        mma_f16_ss_pair(d, a0, b0, idesc, kb > 0);
#pragma unroll
                        for (int k = 1; k < KB / 16; ++k)
                            mma_f16_ss_pair(d, a0 + (uint64_t)(A_MN ? k * 128 : (k >> 2) * 1024 + (k & 3) * 2),
                                            b0 + (uint64_t)(B_MN ? k * 128 : (k >> 2) * 1024 + (k & 3) * 2), idesc, 1u);
                        mma_commit_pair(smem_u32(&bars->empty[ring.slot]));
                    }
                    __syncwarp();
                }
                if (ok && elect_one()) mma_commit_pair(smem_u32(&bars->d_full[buf]));
                __syncwarp();
            }
            if (elect_one()) mma_commit_pair(smem_u32(&bars->drain));           // every MMA issued above completes before tensor memory is freed
            mbar_wait_quiet(smem_u32(&bars->drain), 0u);
        }
    } else {
        const int q = warp & 3, half = warp >= 6 ? 1 : 0;
        const uint32_t lane_base = (uint32_t)(q * 32) << 16;
        uint32_t n_acc = 0;
        for (int64_t item = pair; item < items; item += num_pairs, ++n_acc) {
            int set, m, n;
            item_of(item, set, m, n);
            const int64_t row = (int64_t)m * 256 + rank * 128 + q * 32 + lane, first = row - (lane & 3);
            const uint32_t buf = n_acc & 1u;
            constexpr int SPAN = TILE_N / 2;                 // columns of the result to a group of warps
            const int c_lo = n * TILE_N + half * SPAN;
            const uint32_t taddr = tmem + lane_base + buf * 256 + half * SPAN;
            // GLU_BACK: g and u of 32 columns as they lie in memory (64 bytes of a row at a time, from four lanes), brought a step ahead: the first before the
            // accumulator is waited for, those of the pair's next tile into L2
            uint4 raw[2][4];
            auto fetch = [&](int c0) {
                const bool there = c_lo + c0 + (lane & 3) * 8 < p.cols;
                const __nv_bfloat16* g = p.gate_in + first * p.ld_gate_in + c_lo + c0 + (lane & 3) * 8;
                const __nv_bfloat16* u = p.up_in + first * p.ld_up_in + c_lo + c0 + (lane & 3) * 8;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const bool in = there && first + k < p.rows;
                    raw[0][k] = in ? __ldg(reinterpret_cast<const uint4*>(g + k * p.ld_gate_in)) : make_uint4(0u, 0u, 0u, 0u);
                    raw[1][k] = in ? __ldg(reinterpret_cast<const uint4*>(u + k * p.ld_up_in)) : make_uint4(0u, 0u, 0u, 0u);
                }
            };
            if (MODE == GLU_BACK) {
                fetch(0);
                if (item + num_pairs < items) {
                    int set1, m1, n1;
                    item_of(item + num_pairs, set1, m1, n1);
                    const int64_t row1 = (int64_t)m1 * 256 + rank * 128 + q * 32 + lane;
                    const int col1 = n1 * TILE_N + half * SPAN;
                    if (row1 < p.rows) {
#pragma unroll
                        for (int c = 0; c < SPAN; c += 64) {
                            if (col1 + c >= p.cols) break;
                            prefetch_l2(p.gate_in + row1 * p.ld_gate_in + col1 + c);
                            prefetch_l2(p.up_in + row1 * p.ld_up_in + col1 + c);
                        }
                    }
                }
            }
            bool ok = mbar_wait_cluster(smem_u32(&bars->d_full[buf]), (n_acc >> 1) & 1u, abort_flag, p.timeout_word, TO_EPILOGUE);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            tc_fence_after();
            // 32 columns from c_lo + c0 on, a row to a lane, as bf16: lanes exchange pieces so that a store covers 64 bytes of a row
            auto put = [&](__nv_bfloat16* out, int64_t ld, const float (&v)[32], int c0) {
                uint4 w[4];
                pack_row32(v, w);
                transpose4(w, lane);
                __nv_bfloat16* dst = out + first * ld + c_lo + c0 + (lane & 3) * 8;
                const bool in = c_lo + c0 + (lane & 3) * 8 < p.cols;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (in && first + k < p.rows) *reinterpret_cast<uint4*>(dst + k * ld) = w[k];
            };
#pragma unroll 1
            for (int c0 = 0; c0 < SPAN; c0 += 32) {
                float v[32], u[32];
                if (MODE == GLU_BACK) {
                    float g[32], h[32];
                    transpose4(raw[0], lane);
                    unpack_row32(raw[0], g);
                    transpose4(raw[1], lane);
                    unpack_row32(raw[1], u);
                    if (c0 + 32 < SPAN) fetch(c0 + 32);
                    load_acc(taddr + c0, v);
                    if (c0 + 32 == SPAN) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_leader_tmem(smem_u32(&bars->d_empty[buf]), rank);
                    }
                    by_activation(p.act, [&](auto act) {
#pragma unroll
                        for (int k = 0; k < 32; ++k) {
                            float a, da;
                            activation<act.value>(g[k], a, da);
                            h[k] = a * u[k];
                            g[k] = v[k] * u[k] * da;
                            u[k] = v[k] * a;
                        }
                    });
                    put(p.out, p.ld, g, c0);
                    put(p.out2, p.ld2, u, c0);
                    if (p.out3 != nullptr) put(p.out3, p.ld3, h, c0);
                    continue;
                }
                load_acc(taddr + c0, v);
                if (MODE == GLU) load_acc(taddr + 128 + c0, u);
                if (c0 + 32 == SPAN) {                       // this warp's share of the accumulator is read
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_leader_tmem(smem_u32(&bars->d_empty[buf]), rank);
                }
                if (MODE == GLU) {
                    if (p.out2 != nullptr) { put(p.out2, p.ld2, v, c0); put(p.out3, p.ld3, u, c0); }
                    by_activation(p.act, [&](auto act) {
#pragma unroll
                        for (int k = 0; k < 32; ++k) {
                            float a, da;
                            activation<act.value>(v[k], a, da);
                            v[k] = a * u[k];
                        }
                    });
                    put(p.out, p.ld, v, c0);
                } else {
                    put(set ? p.out2 : p.out, set ? p.ld2 : p.ld, v, c0);
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) pair_drained(&bars->drain);
    cluster_sync_all();
    if (warp == 1) { tc_fence_after(); tmem_dealloc_pair(tmem, 512); }
    cluster_sync_all();                                      // neither CTA of the pair is gone before both have given their half back
}

template <int MODE, bool A_MN, bool B_MN>
qless_status launch_gemm(const char* name, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& a2, const CUtensorMap& b2, const GemmParams& p, cudaStream_t st)
{
    const size_t smem = 1024 + STAGES * 2 * HALF + sizeof(Bars);
    QLESS_CUDA_TRY((allow_full_smem<ffn_gemm_kernel<MODE, A_MN, B_MN>>()));
    const int64_t items = (int64_t)((p.rows + 255) / 256) * ((p.cols + (MODE == GLU ? 127 : 255)) / (MODE == GLU ? 128 : 256)) * p.sets;
    const int64_t grid = std::min<int64_t>(sm_count() / 2 * 2, 2 * items);
    ProfileScope ps(name, st);
    ffn_gemm_kernel<MODE, A_MN, B_MN><<<dim3((unsigned)grid), dim3(NTHREADS), smem, st>>>(a, b, a2, b2, p);
    QLESS_CUDA_TRY(cudaGetLastError());
    count_launches(1);
    return QLESS_OK;
}

// Rows of 64 columns x 128: the box of both operands of a stage, read along or across the contraction.
qless_status map(CUtensorMap* m, const void* p, int64_t cols, int64_t rows, int64_t ld)
{
    return make_tmap_2d_sw128(m, p, 2, (uint64_t)cols, (uint64_t)rows, (uint64_t)ld * 2, 64, 128);
}

}  // namespace

#define QLESS_STEP(expr)                         \
    do {                                         \
        const qless_status s__ = (expr);         \
        if (s__ != QLESS_OK) return s__;         \
    } while (0)

size_t ffn_workspace(int64_t tokens, int32_t width, int32_t inner, bool backward, bool weights)
{
    size_t total = 0;
    if (tokens == 0) return total;
    if (weights) total += align_up((size_t)tokens * inner * 2, 256);      // h
    if (few_tokens(tokens)) total += few_workspace(tokens, width, inner, backward);
    return total;
}

qless_status launch_ffn_forward(const FfnArgs& a, uint8_t* ws, unsigned int* timeout_word, cudaStream_t st)
{
    if (few_tokens(a.tokens)) return launch_few_forward(a, ws, timeout_word, st);
    const int32_t T = (int32_t)a.tokens;
    CUtensorMap x, wg, wu, wd, h;
    QLESS_STEP(map(&x, a.x, a.width, T, a.ld_x));
    QLESS_STEP(map(&wg, a.w_gate, a.width, a.inner, a.ld_wg));
    QLESS_STEP(map(&wu, a.w_up, a.width, a.inner, a.ld_wu));
    QLESS_STEP(map(&wd, a.w_down, a.inner, a.width, a.ld_wd));
    QLESS_STEP(map(&h, a.hidden, a.inner, T, a.ld_hidden));
    GemmParams p{};
    p.rows = T; p.cols = a.inner; p.kblocks = p.kswitch = (a.width + KB - 1) / KB; p.sets = 1; p.act = a.act; p.timeout_word = timeout_word;
    p.out = reinterpret_cast<__nv_bfloat16*>(a.hidden); p.out2 = reinterpret_cast<__nv_bfloat16*>(a.gate); p.out3 = reinterpret_cast<__nv_bfloat16*>(a.up);
    p.ld = a.ld_hidden; p.ld2 = a.ld_gate; p.ld3 = a.ld_up;
    QLESS_STEP((launch_gemm<GLU, false, false>("ffn_glu", x, wg, x, wu, p, st)));
    GemmParams o{};
    o.rows = T; o.cols = a.width; o.kblocks = o.kswitch = (a.inner + KB - 1) / KB; o.sets = 1; o.timeout_word = timeout_word;
    o.out = reinterpret_cast<__nv_bfloat16*>(a.out); o.ld = a.ld_out;
    return launch_gemm<OUT, false, false>("ffn_down", h, wd, h, wd, o, st);
}

qless_status launch_ffn_backward(const FfnArgs& a, uint8_t* ws, unsigned int* timeout_word, cudaStream_t st)
{
    const bool weights = a.dw_gate != nullptr || a.dw_up != nullptr || a.dw_down != nullptr;
    __nv_bfloat16* hidden = a.dw_down != nullptr ? reinterpret_cast<__nv_bfloat16*>(ws) : nullptr;
    if (weights) ws += align_up((size_t)a.tokens * a.inner * 2, 256);
    const int32_t T = (int32_t)a.tokens;
    CUtensorMap dy, x, wg, wu, wd, dg, du, h;
    QLESS_STEP(map(&dy, a.dy, a.width, T, a.ld_dy));
    QLESS_STEP(map(&wg, a.w_gate, a.width, a.inner, a.ld_wg));
    QLESS_STEP(map(&wu, a.w_up, a.width, a.inner, a.ld_wu));
    QLESS_STEP(map(&wd, a.w_down, a.inner, a.width, a.ld_wd));
    QLESS_STEP(map(&dg, a.gate, a.inner, T, a.ld_gate));
    QLESS_STEP(map(&du, a.up, a.inner, T, a.ld_up));
    if (few_tokens(a.tokens)) {
        QLESS_STEP(launch_few_backward(a, hidden, ws, timeout_word, st));
    } else {
        GemmParams p{};
        p.rows = T; p.cols = a.inner; p.kblocks = p.kswitch = (a.width + KB - 1) / KB; p.sets = 1; p.act = a.act; p.timeout_word = timeout_word;
        p.gate_in = reinterpret_cast<const __nv_bfloat16*>(a.gate_in); p.up_in = reinterpret_cast<const __nv_bfloat16*>(a.up_in);
        p.ld_gate_in = a.ld_gate_in; p.ld_up_in = a.ld_up_in;
        p.out = reinterpret_cast<__nv_bfloat16*>(a.gate); p.out2 = reinterpret_cast<__nv_bfloat16*>(a.up); p.out3 = hidden;
        p.ld = a.ld_gate; p.ld2 = a.ld_up; p.ld3 = a.inner;
        QLESS_STEP((launch_gemm<GLU_BACK, false, true>("ffn_glu_back", dy, wd, dy, wd, p, st)));
        if (a.out != nullptr) {
            GemmParams o{};
            o.rows = T; o.cols = a.width; o.kswitch = (a.inner + KB - 1) / KB; o.kblocks = 2 * o.kswitch; o.sets = 1; o.timeout_word = timeout_word;
            o.out = reinterpret_cast<__nv_bfloat16*>(a.out); o.ld = a.ld_out;
            QLESS_STEP((launch_gemm<OUT, false, true>("ffn_grad_x", dg, wg, du, wu, o, st)));
        }
    }
    if (!weights) return QLESS_OK;
    const int32_t kb = (T + KB - 1) / KB;
    if (a.dw_down != nullptr) {
        QLESS_STEP(map(&h, hidden, a.inner, T, a.inner));
        GemmParams o{};
        o.rows = a.width; o.cols = a.inner; o.kblocks = o.kswitch = kb; o.sets = 1; o.timeout_word = timeout_word;
        o.out = reinterpret_cast<__nv_bfloat16*>(a.dw_down); o.ld = a.ld_dwd;
        QLESS_STEP((launch_gemm<OUT, true, true>("ffn_grad_w", dy, h, dy, h, o, st)));
    }
    if (a.dw_gate != nullptr || a.dw_up != nullptr) {
        QLESS_STEP(map(&x, a.x, a.width, T, a.ld_x));
        const bool both = a.dw_gate != nullptr && a.dw_up != nullptr;
        const CUtensorMap& left = a.dw_gate != nullptr ? dg : du;
        GemmParams o{};
        o.rows = a.inner; o.cols = a.width; o.kblocks = o.kswitch = kb; o.sets = both ? 2 : 1; o.timeout_word = timeout_word;
        o.out = reinterpret_cast<__nv_bfloat16*>(a.dw_gate != nullptr ? a.dw_gate : a.dw_up); o.ld = a.dw_gate != nullptr ? a.ld_dwg : a.ld_dwu;
        o.out2 = reinterpret_cast<__nv_bfloat16*>(a.dw_up); o.ld2 = a.ld_dwu;
        QLESS_STEP((launch_gemm<OUT, true, true>("ffn_grad_w", left, x, du, x, o, st)));
    }
    return QLESS_OK;
}

}  // namespace qless
