// Causal attention over packed sequences with grouped heads: the backward pass.
//
//   p_ij = e^(scale <q_i, k_j> - lse_i),  dp_ij = <do_i, v_j>,  delta_i = <do_i, o_i>,  ds_ij = p_ij (dp_ij - delta_i)
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i,   dv_j = sum_i p_ij do_i   (i over the rows and the heads that share key head j)
//
// Two kernels, each with its sums in tensor memory from the first product to the last: one owns a tile of query rows and walks over the keys
// (dq, and delta for the other), one owns a tile of keys and walks over the query rows of every head of its group (dk, dv). Scores and dp are
// computed in both: seven products of a tile instead of five, and in return no partial dq is added up in memory, nothing is
// joined by atomics, and the same inputs give the same bits.
//
// dq kernel, tensor memory: S twice (of this tile of keys and the next), dp, dq: 4 x 128 columns; ds, rounded to bf16, replaces S.
// dk/dv kernel: S^T = K Q^T and dp^T = V dO^T, so that P^T and dS^T are left operands of the products that follow and stay in tensor memory
// (rounded to bf16 in the place of S^T and dp^T), and dv, dk: 4 x 128 columns. While the threads take exponentials of one tile the tensor core
// works on dp and dk, while they form ds it works on dv and the next scores.
// Sixteen warps do the arithmetic, each 32 rows by a quarter of the columns; warp 0 brings tiles by TMA, warp 1 issues products, warps 2 and 3 bring
// lse and delta of the query rows (dk/dv kernel).
// P and ds are rounded to bf16 (2^-9 of each, independent of each other); exponentials, differences and sums are fp32.
// Bound: 128 x 128 scores cost three (dq) and four products of 512 clocks (head_dim 128) and 1024 clocks of the special-function units in each kernel.
#include <algorithm>

#include "attention_common.cuh"

namespace qless {

using namespace attn;

namespace {

constexpr int NTHREADS = 640, MAX_STAGES = 10;

// Columns of step s (16 rows of the contraction) of a left operand in tensor memory that four groups of warps wrote, each over the first half of its own 32 columns.
__device__ __forceinline__ constexpr uint32_t quarter_column(int s) { return (uint32_t)((s >> 1) * 32 + (s & 1) * 8); }

struct QueryParams {
    TileTable table;
    const __nv_bfloat16* out; const __nv_bfloat16* dout;
    const float* lse; float* delta;
    __nv_bfloat16* dq;
    int64_t ld_out, ld_dout, ld_dq;
    int32_t packs, pack, group, heads, head_dim, stages;
    int64_t items;
    float scale, scale_log2;
    unsigned int* timeout_word;
};

struct __align__(8) QueryBars {
    uint64_t q_full, q_empty, full[MAX_STAGES], empty[MAX_STAGES], s_full[2], dp_full, ds_ready, dq_full, delta_ready, drain;
    uint32_t tmem_base, abort_flag;
    float part[2][4][TILE];                 // quarters of delta, of an item and the next
};

template <int DB>
__global__ void __launch_bounds__(NTHREADS, 1)
attention_dq_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_do, const __grid_constant__ CUtensorMap tm_k,
                    const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ QueryParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    constexpr int OP = DB * 16384;
    uint8_t* q_smem = smem;                                  // queries, then the gradient of their outputs
    uint8_t* ring_smem = smem + 2 * OP;
    const uint32_t nS = (uint32_t)p.stages;
    QueryBars* bars = reinterpret_cast<QueryBars*>(ring_smem + (size_t)nS * OP);
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tok = TILE / p.pack;

    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&bars->q_full), 1); mbar_init(smem_u32(&bars->q_empty), 1);
        for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&bars->s_full[i]), 1);
        for (uint32_t i = 0; i < MAX_STAGES; ++i) { mbar_init(smem_u32(&bars->full[i]), 1); mbar_init(smem_u32(&bars->empty[i]), 1); }
        mbar_init(smem_u32(&bars->dp_full), 1); mbar_init(smem_u32(&bars->ds_ready), 16); mbar_init(smem_u32(&bars->dq_full), 1);
        mbar_init(smem_u32(&bars->delta_ready), 16);
        mbar_init(smem_u32(&bars->drain), 1);
        bars->abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tm_q); prefetch_tmap(&tm_do); prefetch_tmap(&tm_k); prefetch_tmap(&tm_v);
    }
    if (warp == 1) { tmem_alloc(smem_u32(&bars->tmem_base), 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;                   // S (ds) at 0 and 128, dp at 256, dq at 384
    ahead_wait();
    ahead_release();

    auto warp_wait = [&](uint64_t* bar, uint32_t parity, uint32_t code) -> bool {
        const bool w = mbar_wait(smem_u32(bar), parity, abort_flag, p.timeout_word, code);
        return __all_sync(0xFFFFFFFFu, w);
    };
    struct Work { AttnTile t; int head0, kv, n; };
    auto work_of = [&](int64_t item) {
        Work w;
        const int i = (int)(item / p.packs), c = (int)(item - (int64_t)i * p.packs);
        w.t = tile_at(p.table, i);
        w.head0 = c * p.pack; w.kv = w.head0 / p.group;
        w.n = (min(w.t.at + tok, w.t.len) + TILE - 1) / TILE;
        return w;
    };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 0) {
            Ring ring;
            uint32_t it = 0, q_uses = 0;
            bool ok = true;
            auto load = [&](const CUtensorMap* map, int kv, int row) {
                if (!warp_wait(&bars->empty[ring.slot], ring.parity ^ 1u, TO_PRODUCER)) { ok = false; return; }
                if (elect_one()) {
                    const uint32_t full = smem_u32(&bars->full[ring.slot]), dst = smem_u32(ring_smem + (size_t)ring.slot * OP);
                    mbar_arrive_expect_tx(full, OP);
#pragma unroll
                    for (int b = 0; b < DB; ++b) tma_load_3d(dst + b * 16384, map, full, b * 64, kv, row);
                }
                __syncwarp();
                ring.next(nS); ++it;
            };
            for (int64_t item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
                const Work w = work_of(item);
                if (!warp_wait(&bars->q_empty, (q_uses++ & 1u) ^ 1u, TO_PRODUCER)) { ok = false; break; }
                if (elect_one()) {
                    const uint32_t full = smem_u32(&bars->q_full), dst = smem_u32(q_smem);
                    mbar_arrive_expect_tx(full, 2 * OP);
#pragma unroll
                    for (int b = 0; b < DB; ++b) {
                        tma_load_3d(dst + b * 16384, &tm_q, full, b * 64, w.head0, w.t.t0 + w.t.at);
                        tma_load_3d(dst + OP + b * 16384, &tm_do, full, b * 64, w.head0, w.t.t0 + w.t.at);
                    }
                }
                __syncwarp();
                for (int j = 0; j < w.n && ok; ++j) {
                    load(&tm_k, w.kv, w.t.t0 + j * TILE);
                    if (ok) load(&tm_v, w.kv, w.t.t0 + j * TILE);
                }
            }
            if (!ok)
                for (uint32_t j = it > nS ? it - nS : 0u; j < it; ++j)
                    if (!mbar_wait_quiet(smem_u32(&bars->full[j % nS]), (j / nS) & 1u, 1u << 14)) break;
        } else if (warp == 1) {
            const uint32_t n_d = (uint32_t)((p.head_dim + 15) / 16 * 16), steps = n_d / 16;
            const uint32_t idesc_s = make_idesc(1, 1, 1, 128, 128), idesc_q = make_idesc(1, 1, 1, 128, n_d) | IDESC_B_MN;
            Ring ring;
            uint32_t q_uses = 0, ds_uses = 0, s_uses = 0;
            bool ok = true;
            auto product = [&](uint32_t d, const uint8_t* a_op, const uint8_t* b_op) {
                const uint64_t a = make_smem_desc_sw128(smem_u32(a_op)), b = make_smem_desc_sw128(smem_u32(b_op));
                for (uint32_t k = 0; k < steps; ++k) {
                    const uint64_t off = (uint64_t)((k >> 2) * 1024 + (k & 3) * 2);
                    mma_f16_ss(d, a + off, b + off, idesc_s, k > 0);
                }
            };
            for (int64_t item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
                const Work w = work_of(item);
                if (!warp_wait(&bars->q_full, q_uses++ & 1u, TO_MMA)) { ok = false; break; }
                Ring k = ring, v;                            // stages of keys and values of tile j
                v = k; v.next(nS);
                auto scores = [&](const Ring& at, int j) -> bool {      // keys behind the sequence's end become zeros: they meet ds = 0 in dq
                    if (!warp_wait(&bars->full[at.slot], at.parity, TO_MMA)) return false;
                    uint8_t* op = ring_smem + (size_t)at.slot * OP;
                    if (w.t.len - j * TILE < TILE) zero_rows(op, DB, w.t.len - j * TILE, lane);
                    tc_fence_after();
                    if (elect_one()) {
                        product(tmem + ((s_uses + j) & 1u) * 128, q_smem, op);
                        mma_commit(smem_u32(&bars->s_full[(s_uses + j) & 1u]));
                    }
                    __syncwarp();
                    return true;
                };
                auto dps = [&](const Ring& at, bool last) -> bool {
                    if (!warp_wait(&bars->full[at.slot], at.parity, TO_MMA)) return false;
                    tc_fence_after();
                    if (elect_one()) {
                        product(tmem + 256, q_smem + OP, ring_smem + (size_t)at.slot * OP);
                        mma_commit(smem_u32(&bars->dp_full));
                        mma_commit(smem_u32(&bars->empty[at.slot]));
                        if (last) mma_commit(smem_u32(&bars->q_empty));
                    }
                    __syncwarp();
                    return true;
                };
                ok = scores(k, 0) && dps(v, w.n == 1);
                for (int j = 0; j < w.n && ok; ++j) {
                    Ring k1 = v, v1;
                    k1.next(nS); v1 = k1; v1.next(nS);
                    if (j + 1 < w.n && !scores(k1, j + 1)) { ok = false; break; }
                    if (!warp_wait(&bars->ds_ready, ds_uses++ & 1u, TO_MMA)) { ok = false; break; }
                    if (j + 1 < w.n && !dps(v1, j + 2 == w.n)) { ok = false; break; }
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t b = make_smem_desc_mn_sw128(smem_u32(ring_smem + (size_t)k.slot * OP), 16384);
                        const uint32_t a = tmem + ((s_uses + j) & 1u) * 128;
#pragma unroll
                        for (int s = 0; s < 8; ++s) mma_f16_ts(tmem + 384, a + quarter_column(s), b + (uint64_t)(s * 128), idesc_q, j > 0 || s > 0);
                        mma_commit(smem_u32(&bars->empty[k.slot]));
                        if (j + 1 == w.n) mma_commit(smem_u32(&bars->dq_full));
                    }
                    __syncwarp();
                    k = k1; v = v1;
                }
                ring = k;                                    // (behind the last tile's)
                s_uses += w.n;
            }
            if (elect_one()) mma_commit(smem_u32(&bars->drain));
            __syncwarp();
            mbar_wait_quiet(smem_u32(&bars->drain), 0u);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        const int part = (warp >> 2) - 1, r = (warp & 3) * 32 + lane;      // which quarter of the columns
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const int my_tok = r / p.pack, my_head = r % p.pack;
        uint32_t s_uses = 0, dp_uses = 0, dq_uses = 0;       // (dq_uses: items so far)
        bool ok = true;
        for (int64_t item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
            const Work w = work_of(item);
            const int at = w.t.at + my_tok;
            const bool there = at < w.t.len;
            const int64_t token = w.t.t0 + at;
            const int head = w.head0 + my_head;
            float delta = 0.0f, off = 0.0f;
            if (there) {
                const __nv_bfloat16* o = p.out + token * p.ld_out + (int64_t)head * p.head_dim;
                const __nv_bfloat16* d = p.dout + token * p.ld_dout + (int64_t)head * p.head_dim;
                float acc[2] = {0.0f, 0.0f};
#pragma unroll 4
                for (int c = part * 8; c < p.head_dim; c += 32) {
                    float a[8], b[8];
                    unpack_bf16(__ldg(reinterpret_cast<const uint4*>(o + c)), a);
                    unpack_bf16(__ldg(reinterpret_cast<const uint4*>(d + c)), b);
#pragma unroll
                    for (int k = 0; k < 8; ++k) acc[k & 1] = fmaf(a[k], b[k], acc[k & 1]);
                }
                delta = acc[0] + acc[1];
                off = p.lse[token * p.heads + head] * LOG2E;
            }
            // The quarters meet through an mbarrier, whose waits end (a block-wide barrier would wait for warps that gave up). An item's places are
            // written again two items later, when every warp has arrived for the item between.
            bars->part[dq_uses & 1u][part][r] = delta;
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars->delta_ready));
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->delta_ready), dq_uses & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
            if (!ok) break;
            const float (*quarters)[TILE] = bars->part[dq_uses & 1u];
            delta = (quarters[0][r] + quarters[1][r]) + (quarters[2][r] + quarters[3][r]);
            if (there && part == 0) p.delta[token * p.heads + head] = delta;
            for (int j = 0; j < w.n; ++j) {
                const uint32_t buf = s_uses & 1u, s_addr = tmem + lanes + buf * 128 + part * 32;
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->s_full[buf]), (s_uses >> 1) & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
                if (!ok) break;
                ++s_uses;
                tc_fence_after();
                uint32_t s[32], dp[32], e[16];
                tmem_ld_x32(s_addr, s);
                tmem_wait_ld();
                const int lim = at - j * TILE - part * 32;   // this row's last key among the 32
#pragma unroll
                for (int k = 0; k < 32; ++k) s[k] = __float_as_uint(ex2(fmaf(__uint_as_float(s[k]), p.scale_log2, -off)));
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->dp_full), dp_uses++ & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
                if (!ok) break;
                tc_fence_after();
                tmem_ld_x32(tmem + lanes + 256 + part * 32, dp);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 32; ++k) dp[k] = __float_as_uint(__uint_as_float(s[k]) * (__uint_as_float(dp[k]) - delta));
                if (j * TILE + TILE - 1 > w.t.at) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) if (k > lim) dp[k] = 0u;
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) e[k] = pack_bf16(__uint_as_float(dp[2 * k]), __uint_as_float(dp[2 * k + 1]));
                tmem_st_x16(s_addr, e);                      // over this quarter's own scores
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars->ds_ready));
            }
            if (!ok) break;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->dq_full), dq_uses++ & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
            if (!ok) break;
            tc_fence_after();
            const int row0 = (warp & 3) * 32;
            auto where = [&](int i) -> __nv_bfloat16* {
                const int rr = row0 + i, a = w.t.at + rr / p.pack;
                return a < w.t.len ? p.dq + (int64_t)(w.t.t0 + a) * p.ld_dq + (int64_t)(w.head0 + rr % p.pack) * p.head_dim : nullptr;
            };
#pragma unroll 1
            for (int c = part * 32; c < p.head_dim; c += 128) {
                uint32_t o[32];
                float f[32];
                tmem_ld_x32(tmem + lanes + 384 + c, o);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 32; ++k) f[k] = __uint_as_float(o[k]) * p.scale;
                store_rows32(f, c, p.head_dim, lane, where);
            }
            tc_fence_before();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, 512); }
}

struct KeyParams {
    TileTable table;
    const float* lse; const float* delta;
    __nv_bfloat16* dk; __nv_bfloat16* dv;
    int64_t ld_dk, ld_dv;
    int32_t kv_heads, pack, group, heads, head_dim;
    int64_t items;
    float scale, scale_log2;
    unsigned int* timeout_word;
};

constexpr int KEY_STAGES = 2;
struct __align__(16) KeyBars {
    float lse[KEY_STAGES][TILE], delta[KEY_STAGES][TILE];      // of each query row: lse times log2 e, delta
    uint64_t kv_full, kv_empty, full[KEY_STAGES], empty[KEY_STAGES], stat_full[KEY_STAGES], stat_empty[KEY_STAGES], s_full, dp_full, p_ready, ds_ready, done, drain;
    uint32_t tmem_base, abort_flag;
};

template <int DB>
__global__ void __launch_bounds__(NTHREADS, 1)
attention_dkv_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_do, const __grid_constant__ CUtensorMap tm_k,
                     const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ KeyParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    constexpr int OP = DB * 16384;
    uint8_t* kv_smem = smem;                                 // keys, values
    uint8_t* ring_smem = smem + 2 * OP;                      // queries and the gradient of their outputs, KEY_STAGES times
    KeyBars* bars = reinterpret_cast<KeyBars*>(ring_smem + KEY_STAGES * 2 * OP);
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tok = TILE / p.pack, passes = p.group / p.pack;

    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&bars->kv_full), 1); mbar_init(smem_u32(&bars->kv_empty), 1);
        for (int i = 0; i < KEY_STAGES; ++i) {
            mbar_init(smem_u32(&bars->full[i]), 1); mbar_init(smem_u32(&bars->empty[i]), 1);
            mbar_init(smem_u32(&bars->stat_full[i]), 2); mbar_init(smem_u32(&bars->stat_empty[i]), 16);
        }
        mbar_init(smem_u32(&bars->s_full), 1); mbar_init(smem_u32(&bars->dp_full), 1); mbar_init(smem_u32(&bars->done), 1);
        mbar_init(smem_u32(&bars->p_ready), 16); mbar_init(smem_u32(&bars->ds_ready), 16); mbar_init(smem_u32(&bars->drain), 1);
        bars->abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tm_q); prefetch_tmap(&tm_do); prefetch_tmap(&tm_k); prefetch_tmap(&tm_v);
    }
    if (warp == 1) { tmem_alloc(smem_u32(&bars->tmem_base), 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;                   // S^T (P^T) at 0, dp^T (dS^T) at 128, dv at 256, dk at 384
    ahead_wait();
    ahead_release();

    auto warp_wait = [&](uint64_t* bar, uint32_t parity, uint32_t code) -> bool {
        const bool w = mbar_wait(smem_u32(bar), parity, abort_flag, p.timeout_word, code);
        return __all_sync(0xFFFFFFFFu, w);
    };
    // loops: for every pass over `pack` heads of the group, the tiles of queries from the one that holds the first key's token on
    struct Work { AttnTile t; int kv, first, per, n; };
    auto work_of = [&](int64_t item) {
        Work w;
        const int i = (int)(item / p.kv_heads);
        w.kv = (int)(item - (int64_t)i * p.kv_heads);
        w.t = tile_at(p.table, i);
        w.first = w.t.at / tok;
        w.per = (w.t.len + tok - 1) / tok - w.first;
        w.n = w.per * passes;
        return w;
    };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 0) {
            Ring ring;
            uint32_t it = 0, kv_uses = 0;
            bool ok = true;
            for (int64_t item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
                const Work w = work_of(item);
                if (!warp_wait(&bars->kv_empty, (kv_uses++ & 1u) ^ 1u, TO_PRODUCER)) { ok = false; break; }
                if (elect_one()) {
                    const uint32_t full = smem_u32(&bars->kv_full), dst = smem_u32(kv_smem);
                    mbar_arrive_expect_tx(full, 2 * OP);
#pragma unroll
                    for (int b = 0; b < DB; ++b) {
                        tma_load_3d(dst + b * 16384, &tm_k, full, b * 64, w.kv, w.t.t0 + w.t.at);
                        tma_load_3d(dst + OP + b * 16384, &tm_v, full, b * 64, w.kv, w.t.t0 + w.t.at);
                    }
                }
                __syncwarp();
                int head0 = w.kv * p.group, i = w.first, left = w.per;
                for (int j = 0; j < w.n; ++j, ++it, ring.next(KEY_STAGES)) {
                    if (!warp_wait(&bars->empty[ring.slot], ring.parity ^ 1u, TO_PRODUCER)) { ok = false; break; }
                    if (elect_one()) {
                        const uint32_t full = smem_u32(&bars->full[ring.slot]), dst = smem_u32(ring_smem + (size_t)ring.slot * 2 * OP);
                        mbar_arrive_expect_tx(full, 2 * OP);
#pragma unroll
                        for (int b = 0; b < DB; ++b) {
                            tma_load_3d(dst + b * 16384, &tm_q, full, b * 64, head0, w.t.t0 + i * tok);
                            tma_load_3d(dst + OP + b * 16384, &tm_do, full, b * 64, head0, w.t.t0 + i * tok);
                        }
                    }
                    __syncwarp();
                    ++i;
                    if (--left == 0) { left = w.per; i = w.first; head0 += p.pack; }
                }
            }
            if (!ok)
                for (uint32_t j = it > KEY_STAGES ? it - KEY_STAGES : 0u; j < it; ++j)
                    if (!mbar_wait_quiet(smem_u32(&bars->full[j % KEY_STAGES]), (j / KEY_STAGES) & 1u, 1u << 14)) break;
        } else if (warp == 1) {
            const uint32_t n_d = (uint32_t)((p.head_dim + 15) / 16 * 16), steps = n_d / 16;
            const uint32_t idesc_s = make_idesc(1, 1, 1, 128, 128), idesc_g = make_idesc(1, 1, 1, 128, n_d) | IDESC_B_MN;
            Ring ring;
            uint32_t kv_uses = 0, p_uses = 0, ds_uses = 0;
            bool ok = true;
            auto product = [&](uint32_t d, const uint8_t* a_op, const uint8_t* b_op) {
                const uint64_t a = make_smem_desc_sw128(smem_u32(a_op)), b = make_smem_desc_sw128(smem_u32(b_op));
                for (uint32_t k = 0; k < steps; ++k) {
                    const uint64_t off = (uint64_t)((k >> 2) * 1024 + (k & 3) * 2);
                    mma_f16_ss(d, a + off, b + off, idesc_s, k > 0);
                }
            };
            auto gradient = [&](uint32_t d, uint32_t a, const uint8_t* b_op, bool more) {
                const uint64_t b = make_smem_desc_mn_sw128(smem_u32(b_op), 16384);
#pragma unroll
                for (int s = 0; s < 8; ++s) mma_f16_ts(d, a + quarter_column(s), b + (uint64_t)(s * 128), idesc_g, more || s > 0);
            };
            for (int64_t item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
                const Work w = work_of(item);
                if (!warp_wait(&bars->kv_full, kv_uses++ & 1u, TO_MMA)) { ok = false; break; }
                int i = w.first, left = w.per;
                // The tile's queries have arrived; rows behind the sequence's end become zeros in both operands (they meet P = dS = 0).
                auto arrived = [&](const Ring& at) -> bool {
                    if (!warp_wait(&bars->full[at.slot], at.parity, TO_MMA)) return false;
                    const int have = (w.t.len - i * tok) * p.pack;
                    uint8_t* op = ring_smem + (size_t)at.slot * 2 * OP;
                    if (have < TILE) zero_rows(op, 2 * DB, have, lane);
                    ++i;
                    if (--left == 0) { left = w.per; i = w.first; }
                    tc_fence_after();
                    return true;
                };
                if (!arrived(ring)) { ok = false; break; }
                if (elect_one()) {
                    const uint8_t* op = ring_smem + (size_t)ring.slot * 2 * OP;
                    product(tmem, kv_smem, op);
                    mma_commit(smem_u32(&bars->s_full));
                    product(tmem + 128, kv_smem + OP, op + OP);
                    mma_commit(smem_u32(&bars->dp_full));
                    if (w.n == 1) mma_commit(smem_u32(&bars->kv_empty));
                }
                __syncwarp();
                for (int j = 0; j < w.n && ok; ++j) {
                    Ring next = ring;
                    next.next(KEY_STAGES);
                    const bool more = j + 1 < w.n;
                    const uint8_t* op = ring_smem + (size_t)ring.slot * 2 * OP;
                    const uint8_t* op1 = ring_smem + (size_t)next.slot * 2 * OP;
                    if (!warp_wait(&bars->p_ready, p_uses++ & 1u, TO_MMA)) { ok = false; break; }
                    tc_fence_after();
                    if (elect_one()) gradient(tmem + 256, tmem, op + OP, j > 0);
                    __syncwarp();
                    if (more && !arrived(next)) { ok = false; break; }
                    if (more && elect_one()) {
                        product(tmem, kv_smem, op1);
                        mma_commit(smem_u32(&bars->s_full));
                    }
                    __syncwarp();
                    if (!warp_wait(&bars->ds_ready, ds_uses++ & 1u, TO_MMA)) { ok = false; break; }
                    tc_fence_after();
                    if (elect_one()) {
                        gradient(tmem + 384, tmem + 128, op, j > 0);
                        mma_commit(smem_u32(&bars->empty[ring.slot]));
                        if (more) {
                            product(tmem + 128, kv_smem + OP, op1 + OP);
                            mma_commit(smem_u32(&bars->dp_full));
                            if (j + 2 == w.n) mma_commit(smem_u32(&bars->kv_empty));
                        } else {
                            mma_commit(smem_u32(&bars->done));
                        }
                    }
                    __syncwarp();
                    ring = next;
                }
            }
            if (elect_one()) mma_commit(smem_u32(&bars->drain));
            __syncwarp();
            mbar_wait_quiet(smem_u32(&bars->drain), 0u);
        } else {
            Ring ring;
            bool ok = true;
            for (int64_t item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
                const Work w = work_of(item);
                int head0 = w.kv * p.group, i = w.first, left = w.per;
                for (int j = 0; j < w.n; ++j, ring.next(KEY_STAGES)) {
                    float lse[2], delta[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {            // rows behind the end: P = e^(0 - infinity) = 0, dS = 0
                        const int r = (warp - 2) * 64 + h * 32 + lane, at = i * tok + r / p.pack;
                        lse[h] = INFINITY; delta[h] = 0.0f;
                        if (at < w.t.len) {
                            const int64_t row = (int64_t)(w.t.t0 + at) * p.heads + head0 + r % p.pack;
                            lse[h] = p.lse[row] * LOG2E; delta[h] = p.delta[row];
                        }
                    }
                    if (!warp_wait(&bars->stat_empty[ring.slot], ring.parity ^ 1u, TO_PRODUCER)) { ok = false; break; }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int r = (warp - 2) * 64 + h * 32 + lane;
                        bars->lse[ring.slot][r] = lse[h]; bars->delta[ring.slot][r] = delta[h];
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&bars->stat_full[ring.slot]));
                    ++i;
                    if (--left == 0) { left = w.per; i = w.first; head0 += p.pack; }
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        const int part = (warp >> 2) - 1, r = (warp & 3) * 32 + lane;      // which quarter of the columns
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_addr = tmem + lanes + part * 32, dp_addr = s_addr + 128;
        uint32_t uses = 0, done_uses = 0;
        Ring ring;
        bool ok = true;
        for (int64_t item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
            const Work w = work_of(item);
            const int key = w.t.at + r;
            int i = w.first, left = w.per;
            for (int j = 0; j < w.n; ++j, ++uses, ring.next(KEY_STAGES)) {
                // column c of this quarter is query row part * 32 + c: token i * tok + (part * 32 + c) / pack; it sees this row's key from `from` on
                const bool masked = i * tok < w.t.at + TILE - 1;
                const int from = (key - i * tok) * p.pack - part * 32;
                ++i;
                if (--left == 0) { left = w.per; i = w.first; }
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->stat_full[ring.slot]), ring.parity, abort_flag, p.timeout_word, TO_EPILOGUE));
                if (!ok) break;
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->s_full), uses & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
                if (!ok) break;
                tc_fence_after();
                uint32_t s[32], dp[32], e[16];
                tmem_ld_x32(s_addr, s);
                const float4* lse = reinterpret_cast<const float4*>(&bars->lse[ring.slot][part * 32]);
                const float4* delta = reinterpret_cast<const float4*>(&bars->delta[ring.slot][part * 32]);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 32; k += 4) {
                    const float4 l = lse[k / 4];
                    s[k] = __float_as_uint(ex2(fmaf(__uint_as_float(s[k]), p.scale_log2, -l.x)));
                    s[k + 1] = __float_as_uint(ex2(fmaf(__uint_as_float(s[k + 1]), p.scale_log2, -l.y)));
                    s[k + 2] = __float_as_uint(ex2(fmaf(__uint_as_float(s[k + 2]), p.scale_log2, -l.z)));
                    s[k + 3] = __float_as_uint(ex2(fmaf(__uint_as_float(s[k + 3]), p.scale_log2, -l.w)));
                }
                if (masked) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) if (k < from) s[k] = 0u;
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) e[k] = pack_bf16(__uint_as_float(s[2 * k]), __uint_as_float(s[2 * k + 1]));
                tmem_st_x16(s_addr, e);                      // over this quarter's own scores
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars->p_ready));
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->dp_full), uses & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
                if (!ok) break;
                tc_fence_after();
                tmem_ld_x32(dp_addr, dp);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 32; k += 4) {
                    const float4 d = delta[k / 4];
                    dp[k] = __float_as_uint(__uint_as_float(s[k]) * (__uint_as_float(dp[k]) - d.x));
                    dp[k + 1] = __float_as_uint(__uint_as_float(s[k + 1]) * (__uint_as_float(dp[k + 1]) - d.y));
                    dp[k + 2] = __float_as_uint(__uint_as_float(s[k + 2]) * (__uint_as_float(dp[k + 2]) - d.z));
                    dp[k + 3] = __float_as_uint(__uint_as_float(s[k + 3]) * (__uint_as_float(dp[k + 3]) - d.w));
                }
                if (masked) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) if (k < from) dp[k] = 0u;
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) e[k] = pack_bf16(__uint_as_float(dp[2 * k]), __uint_as_float(dp[2 * k + 1]));
                tmem_st_x16(dp_addr, e);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) { mbar_arrive(smem_u32(&bars->ds_ready)); mbar_arrive(smem_u32(&bars->stat_empty[ring.slot])); }
            }
            if (!ok) break;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->done), done_uses++ & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
            if (!ok) break;
            tc_fence_after();
            // two groups of warps have dv, two dk: every other 32 columns each
            const bool is_k = part >= 2;
            __nv_bfloat16* base = is_k ? p.dk : p.dv;
            const int64_t ld = is_k ? p.ld_dk : p.ld_dv;
            const float by = is_k ? p.scale : 1.0f;
            const int row0 = w.t.at + (warp & 3) * 32;
            auto where = [&](int k) -> __nv_bfloat16* {
                return row0 + k < w.t.len ? base + (int64_t)(w.t.t0 + row0 + k) * ld + (int64_t)w.kv * p.head_dim : nullptr;
            };
#pragma unroll 1
            for (int c = (part & 1) * 32; c < p.head_dim; c += 64) {
                uint32_t o[32];
                float f[32];
                tmem_ld_x32(tmem + lanes + 256 + (is_k ? 128 : 0) + c, o);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 32; ++k) f[k] = __uint_as_float(o[k]) * by;
                store_rows32(f, c, p.head_dim, lane, where);
            }
            tc_fence_before();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, 512); }
}

template <int DB>
qless_status launch_backward(const CUtensorMap& q, const CUtensorMap& d, const CUtensorMap& k, const CUtensorMap& v, QueryParams& qp, const KeyParams& kp, cudaStream_t st)
{
    const size_t op = (size_t)DB * 16384, budget = 227 * 1024 - 1024 - sizeof(QueryBars) - 2 * op;
    qp.stages = (int32_t)std::min<size_t>(MAX_STAGES, budget / op);
    const size_t q_smem = 1024 + (2 + qp.stages) * op + sizeof(QueryBars), k_smem = 1024 + (2 + 2 * KEY_STAGES) * op + sizeof(KeyBars);
    { ProfileScope ps("attention_dq", st);
      QLESS_CUDA_TRY((allow_full_smem<attention_dq_kernel<DB>>()));
      QLESS_CUDA_TRY(launch_ahead(attention_dq_kernel<DB>, dim3((unsigned)std::min<int64_t>(qp.items, sm_count())), dim3(NTHREADS), q_smem, st, q, d, k, v, qp)); }
    count_launches(1);
    { ProfileScope ps("attention_dkv", st);
      QLESS_CUDA_TRY((allow_full_smem<attention_dkv_kernel<DB>>()));
      QLESS_CUDA_TRY(launch_ahead(attention_dkv_kernel<DB>, dim3((unsigned)std::min<int64_t>(kp.items, sm_count())), dim3(NTHREADS), k_smem, st, q, d, k, v, kp)); }
    count_launches(1);
    return QLESS_OK;
}

size_t tiles_bytes(int64_t tokens, int64_t n, int64_t rows) { return align_up((size_t)(tokens / rows + n + 1) * sizeof(AttnTile), 256); }

}  // namespace

size_t attention_workspace(int64_t tokens, int64_t n, int32_t heads, int32_t kv_heads, bool backward)
{
    // a sequence has at most one tile that is not full; sequences without tokens have none
    const int64_t seqs = std::min(tokens, n), tok = TILE / attn_pack(heads, kv_heads);
    size_t total = tiles_bytes(tokens, seqs, tok) + 256;
    if (backward) total += tiles_bytes(tokens, seqs, TILE) + align_up((size_t)tokens * heads * 4, 256);
    return total;
}

qless_status launch_attention_backward(const AttnArgs& a, uint8_t* ws, unsigned int* timeout_word, cudaStream_t st)
{
    const int32_t pack = attn_pack(a.heads, a.kv_heads), tok = TILE / pack, packs = a.heads / pack;
    const std::vector<AttnTile> queries = query_tiles(a, tok), keys = key_tiles(a);
    if (queries.empty()) return QLESS_OK;
    const int64_t seqs = std::min(a.tokens, a.n);
    AttnTile* q_list = reinterpret_cast<AttnTile*>(ws);
    AttnTile* k_list = reinterpret_cast<AttnTile*>(ws + tiles_bytes(a.tokens, seqs, tok));
    float* delta = reinterpret_cast<float*>(ws + tiles_bytes(a.tokens, seqs, tok) + tiles_bytes(a.tokens, seqs, TILE));
    QueryParams qp;
    KeyParams kp;
    qless_status s;
    if ((s = put_table(queries, &qp.table, q_list, st)) != QLESS_OK) return s;
    if ((s = put_table(keys, &kp.table, k_list, st)) != QLESS_OK) return s;
    CUtensorMap q, d, k, v;
    if ((s = head_map(&q, a.q, a.ld_q, a.heads, a.head_dim, a.tokens, pack, tok)) != QLESS_OK) return s;
    if ((s = head_map(&d, a.dout, a.ld_dout, a.heads, a.head_dim, a.tokens, pack, tok)) != QLESS_OK) return s;
    if ((s = head_map(&k, a.k, a.ld_k, a.kv_heads, a.head_dim, a.tokens, 1, TILE)) != QLESS_OK) return s;
    if ((s = head_map(&v, a.v, a.ld_v, a.kv_heads, a.head_dim, a.tokens, 1, TILE)) != QLESS_OK) return s;
    qp.out = reinterpret_cast<const __nv_bfloat16*>(a.out_in); qp.dout = reinterpret_cast<const __nv_bfloat16*>(a.dout); qp.lse = a.lse_in; qp.delta = delta;
    qp.dq = reinterpret_cast<__nv_bfloat16*>(a.dq); qp.ld_out = a.ld_out; qp.ld_dout = a.ld_dout; qp.ld_dq = a.ld_dq;
    qp.packs = packs; qp.pack = pack; qp.group = a.heads / a.kv_heads; qp.heads = a.heads; qp.head_dim = a.head_dim;
    qp.items = (int64_t)queries.size() * packs; qp.scale = a.scale; qp.scale_log2 = a.scale * LOG2E; qp.timeout_word = timeout_word;
    kp.lse = a.lse_in; kp.delta = delta; kp.dk = reinterpret_cast<__nv_bfloat16*>(a.dk); kp.dv = reinterpret_cast<__nv_bfloat16*>(a.dv);
    kp.ld_dk = a.ld_dk; kp.ld_dv = a.ld_dv; kp.kv_heads = a.kv_heads; kp.pack = pack; kp.group = qp.group; kp.heads = a.heads; kp.head_dim = a.head_dim;
    kp.items = (int64_t)keys.size() * a.kv_heads; kp.scale = a.scale; kp.scale_log2 = qp.scale_log2; kp.timeout_word = timeout_word;
    return a.head_dim <= 64 ? launch_backward<1>(q, d, k, v, qp, kp, st) : launch_backward<2>(q, d, k, v, qp, kp, st);
}

}  // namespace qless
