// Causal attention over packed sequences with grouped heads: the backward pass.
//
//   p_ij = e^(scale <q_i, k_j> - lse_i),  dp_ij = <do_i, v_j>,  delta_i = <do_i, o_i>,  ds_ij = p_ij (dp_ij - delta_i)
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i,   dv_j = sum_i p_ij do_i   (i over the rows and the heads that share key head j)
//
// Two kernels, each with its sums in tensor memory from the first product to the last: one owns a tile of query rows and walks over the keys
// (dq, and delta for the other), one owns a tile of keys and walks over the query rows of every head of its group (dk, dv). Scores and dp are
// computed in both (seven products of a tile instead of five, and the eighth of kbar below), and in return nothing is joined by atomics and the same inputs
// give the same bits. Where tiles are few and loops long, pieces of a loop leave their sums in memory and a small kernel adds them in order (split_tiles).
//
// delta taken from the output as it was handed on, in bf16, would be off by up to 2^-8 of |do| |o|, and with rows that look at few keys (|o| near |v|, ds small)
// that is more than all other roundings together: errors of 3e-3 to 4.4e-3 of the gradients' norm were seen where 2.4e-3 are due to bf16 operands and
// results (examples of some hundred tokens and more; where a few entries of ds make up a gradient, their roundings do not average: up to 3.4e-3, and as much with an exact
// delta). But sum_j ds_ij = 0 when delta is exact, so the row sum of what is formed with the rough delta, rho_i = sum_j ds_ij (fp32, before rounding), is delta's
// error: the dq kernel also sums kbar_i = sum_j p_ij k_j and returns scale (sum_j ds_ij k_j - rho_i kbar_i), and hands delta_i + rho_i to the other kernel.
//
// dq kernel, tensor memory: S, dp, dq, kbar: 4 x 128 columns; P and ds, rounded to bf16, replace S and dp. While the threads take exponentials of one tile
// the tensor core works on dq and the next dp, while they form ds it works on kbar and the next scores.
// dk/dv kernel, in the same order: S^T = K Q^T and dp^T = V dO^T, so that P^T and dS^T are left operands of the products that follow and stay in
// tensor memory, and dv, dk.
// Sixteen warps do the arithmetic, each 32 rows by a quarter of the columns; warp 0 brings tiles by TMA, warp 1 issues products, warps 2 and 3 bring
// lse and delta of the query rows (dk/dv kernel).
// P and ds are rounded to bf16 (at most 2^-8 of each, independent of each other); exponentials, differences and sums are fp32.
// Bound: 128 x 128 scores cost four products of 512 clocks (head_dim 128) and 1024 clocks of the special-function units in each kernel.
// 32 examples of 16381 tokens in all, 32/8 heads of 128: 281 us (dq) and 196 us (dk, dv); one of 8191 tokens, 16/16 heads of 64: 361 and 314 us. Short examples wait for a
// tile's own chain: tensor pipe 34 and 48 % busy. (S, dp and the two sums fill tensor memory, so neither S nor dp has a second place; without kbar there would be one.)
#include <algorithm>
#include <type_traits>

#include "attention_common.cuh"

namespace qless {

using namespace attn;

namespace {

constexpr int NTHREADS = 640;

// Columns of step s (16 rows of the contraction) of a left operand in tensor memory that four groups of warps wrote, each over the first half of its own 32 columns.
__device__ __forceinline__ constexpr uint32_t quarter_column(int s) { return (uint32_t)((s >> 1) * 32 + (s & 1) * 8); }

// 32 columns of this lane's row of sums, as they are.
__device__ __forceinline__ void put_sums(uint32_t taddr, float* dst)
{
    uint32_t o[32];
    __syncwarp();                                            // (a whole warp's load: lanes may come from stores that some of them did not make)
    tmem_ld_x32(taddr, o);
    tmem_wait_ld();
#pragma unroll
    for (int k = 0; k < 8; ++k)
        reinterpret_cast<float4*>(dst)[k] = make_float4(__uint_as_float(o[4 * k]), __uint_as_float(o[4 * k + 1]), __uint_as_float(o[4 * k + 2]), __uint_as_float(o[4 * k + 3]));
}

struct QueryParams {
    TileTable table;
    const __nv_bfloat16* out; const __nv_bfloat16* dout;
    const float* lse; float* delta;         // (delta is kept negated)
    __nv_bfloat16* dq;
    int64_t ld_out, ld_dout, ld_dq;
    uint32_t items, packs;
    int32_t chunk;                          // > 0: items are pieces of tiles, of so many tiles of keys; a tile of several leaves its sums here:
    float* part; float2* stat;              // [item][row][dq, kbar: 64 DB each]; [item][row]: rho, delta as taken from the output (negated)
    int32_t pack, pack_shift, group, heads, head_dim;
    float scale, scale_log2;
    unsigned int* timeout_word;
};

// Stages: tiles of keys and of values have rings of their own, for a tile of values is done with long before the keys beside it.
template <int DB> struct QueryStages { static constexpr int K = DB == 1 ? 4 : 3, V = DB == 1 ? 3 : 1; };

template <int DB>
struct __align__(16) QueryBars {
    float lse[TILE], delta[TILE];           // of an item's rows, negated: lse times log2 e, delta as taken from the output; at its end rho
    uint64_t q_full[2], q_empty[2], do_full, do_empty, k_full[QueryStages<DB>::K], k_empty[QueryStages<DB>::K], v_full[QueryStages<DB>::V], v_empty[QueryStages<DB>::V];
    uint64_t s_full, dp_full, p_ready, ds_ready, dq_full, stat_full, rho_low, rho_sum, rho_read, drain;
    uint32_t tmem_base, abort_flag;
};

// The roles walk over the same flat sequence of tiles, item after item: queries and dO of the next item are brought, its statistics taken and its first scores
// formed while the last tiles of the one before are worked on.
template <int DB>
__global__ void __launch_bounds__(NTHREADS, 1)
attention_dq_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_do, const __grid_constant__ CUtensorMap tm_k,
                    const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_o, const __grid_constant__ QueryParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    constexpr int OP = DB * 16384;
    constexpr uint32_t KS = QueryStages<DB>::K, VS = QueryStages<DB>::V;
    uint8_t* q_smem = smem;                                  // queries of two items, the gradient of one's outputs
    uint8_t* do_smem = smem + 2 * OP;
    uint8_t* k_smem = smem + 3 * OP;
    uint8_t* v_smem = k_smem + KS * OP;
    QueryBars<DB>* bars = reinterpret_cast<QueryBars<DB>*>(v_smem + VS * OP);
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int tok = TILE >> p.pack_shift;

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&bars->q_full[i]), 1); mbar_init(smem_u32(&bars->q_empty[i]), 1); }
        for (uint32_t i = 0; i < KS; ++i) { mbar_init(smem_u32(&bars->k_full[i]), 1); mbar_init(smem_u32(&bars->k_empty[i]), 1); }
        for (uint32_t i = 0; i < VS; ++i) { mbar_init(smem_u32(&bars->v_full[i]), 1); mbar_init(smem_u32(&bars->v_empty[i]), 1); }
        mbar_init(smem_u32(&bars->rho_low), 8); mbar_init(smem_u32(&bars->rho_sum), 8); mbar_init(smem_u32(&bars->rho_read), 16);
        mbar_init(smem_u32(&bars->s_full), 1); mbar_init(smem_u32(&bars->p_ready), 16);
        mbar_init(smem_u32(&bars->dp_full), 1); mbar_init(smem_u32(&bars->ds_ready), 16); mbar_init(smem_u32(&bars->dq_full), 1);
        mbar_init(smem_u32(&bars->stat_full), 16); mbar_init(smem_u32(&bars->drain), 1);
        mbar_init(smem_u32(&bars->do_full), 1); mbar_init(smem_u32(&bars->do_empty), 1);
        bars->abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tm_q); prefetch_tmap(&tm_do); prefetch_tmap(&tm_k); prefetch_tmap(&tm_v);
    }
    if (warp == 1) { tmem_alloc(smem_u32(&bars->tmem_base), 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;                   // S (P) at 0, dp (ds) at 128, dq at 256, kbar at 384
    ahead_wait();
    ahead_release();

    auto warp_wait = [&](uint64_t* bar, uint32_t parity, uint32_t code) -> bool {
        const bool w = mbar_wait(smem_u32(bar), parity, abort_flag, p.timeout_word, code);
        return __all_sync(0xFFFFFFFFu, w);
    };
    struct Work { AttnTile t; int head0, kv, n; };           // (tiles of keys from t.way on)
    auto loops = [&](const AttnTile& t) { return (min(t.at + tok, t.len) + TILE - 1) / TILE; };
    auto work_of = [&](const Walk& k) {
        Work w;
        w.t = k.tile;
        w.head0 = (int)k.sub * p.pack; w.kv = w.head0 / p.group;
        w.n = loops(w.t) - w.t.way;
        if (p.chunk > 0) w.n = min(p.chunk, w.n);
        return w;
    };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 0) {
            Ring k_ring, v_ring;
            uint32_t items = 0, tiles = 0;
            bool ok = true;
            auto load = [&](const CUtensorMap* map, uint64_t* full_bar, uint8_t* dst_op, int kv, int row) {
                if (elect_one()) {
                    const uint32_t full = smem_u32(full_bar), dst = smem_u32(dst_op);
                    mbar_arrive_expect_tx(full, OP);
#pragma unroll
                    for (int b = 0; b < DB; ++b) tma_load_3d(dst + b * 16384, map, full, b * 64, kv, row);
                }
                __syncwarp();
            };
            for (Walk walk(p.table, p.items, p.packs); walk.more && ok; walk.next(), ++items) {
                const Work w = work_of(walk);
                const uint32_t b2 = items & 1u;
                if (!warp_wait(&bars->q_empty[b2], ((items >> 1) & 1u) ^ 1u, TO_PRODUCER)) { ok = false; break; }
                if (elect_one()) {
                    const uint32_t full = smem_u32(&bars->q_full[b2]), dst = smem_u32(q_smem + b2 * OP);
                    mbar_arrive_expect_tx(full, OP);
#pragma unroll
                    for (int b = 0; b < DB; ++b) tma_load_3d(dst + b * 16384, &tm_q, full, b * 64, w.head0, w.t.t0 + w.t.at);
                }
                __syncwarp();
                for (int j = 0; j < w.n; ++j, ++tiles) {
                    if (!warp_wait(&bars->k_empty[k_ring.slot], k_ring.parity ^ 1u, TO_PRODUCER)) { ok = false; break; }
                    load(&tm_k, &bars->k_full[k_ring.slot], k_smem + (size_t)k_ring.slot * OP, w.kv, w.t.t0 + (w.t.way + j) * TILE);
                    k_ring.next(KS);
                    if (j == 0) {
                        if (!warp_wait(&bars->do_empty, (items & 1u) ^ 1u, TO_PRODUCER)) { ok = false; break; }
                        load(&tm_do, &bars->do_full, do_smem, w.head0, w.t.t0 + w.t.at);
                        // the statistics of the next item's rows come out of L2
                        const uint32_t item = item_of_round(walk.round + 1);
                        if (item < p.items) {
                            const AttnTile t = uniform_tile(walk.after);
                            const int head0 = (int)(item - item / p.packs * p.packs) * p.pack;
                            if (elect_one()) {
#pragma unroll
                                for (int b = 0; b < DB; ++b) { tma_prefetch_3d(&tm_o, b * 64, head0, t.t0 + t.at); tma_prefetch_3d(&tm_do, b * 64, head0, t.t0 + t.at); }
                            }
                            __syncwarp();
                        }
                    }
                    if (!warp_wait(&bars->v_empty[v_ring.slot], v_ring.parity ^ 1u, TO_PRODUCER)) { ok = false; break; }
                    load(&tm_v, &bars->v_full[v_ring.slot], v_smem + (size_t)v_ring.slot * OP, w.kv, w.t.t0 + (w.t.way + j) * TILE);
                    v_ring.next(VS);
                }
            }
            // behind a wait that gave up: what is still on its way arrives before the block leaves
            if (!ok) {
                for (uint32_t i = items > 1 ? items - 1 : 0u; i <= items; ++i) mbar_wait_quiet(smem_u32(&bars->q_full[i & 1u]), (i >> 1) & 1u, 1u << 14);
                if (items > 0) mbar_wait_quiet(smem_u32(&bars->do_full), (items - 1) & 1u, 1u << 14);
                mbar_wait_quiet(smem_u32(&bars->do_full), items & 1u, 1u << 14);
                for (uint32_t i = tiles > KS ? tiles - KS : 0u; i <= tiles; ++i) mbar_wait_quiet(smem_u32(&bars->k_full[i % KS]), (i / KS) & 1u, 1u << 14);
                for (uint32_t i = tiles > VS ? tiles - VS : 0u; i < tiles; ++i) mbar_wait_quiet(smem_u32(&bars->v_full[i % VS]), (i / VS) & 1u, 1u << 14);
            }
        } else if (warp == 1) {
            const uint32_t n_d = (uint32_t)((p.head_dim + 15) / 16 * 16), steps = n_d / 16;
            const uint32_t idesc_s = make_idesc(1, 1, 1, 128, 128), idesc_q = make_idesc(1, 1, 1, 128, n_d) | IDESC_B_MN;
            auto product = [&](uint32_t d, const uint8_t* a_op, const uint8_t* b_op) {
                const uint64_t a = make_smem_desc_sw128(smem_u32(a_op)), b = make_smem_desc_sw128(smem_u32(b_op));
#pragma unroll
                for (uint32_t k = 0; k < 4 * DB; ++k) {
                    const uint64_t off = (uint64_t)((k >> 2) * 1024 + (k & 3) * 2);
                    if (k < steps) mma_f16_ss(d, a + off, b + off, idesc_s, k > 0);
                }
            };
            // A place in the sequence of tiles; scores and dp run one tile ahead of the sums.
            struct Place { Work w; int j; uint32_t items; };
            Ring k_ring, k_use, v_ring;                      // keys for the scores, for dq; values
            uint32_t tiles = 0;
            bool ok = true;
            Walk walk(p.table, p.items, p.packs);
            Place ahead;
            ahead.j = 0; ahead.items = 0;
            if (walk.more) ahead.w = work_of(walk);
            auto scores = [&]() -> bool {                    // of the tile at `ahead`: keys behind the sequence's end become zeros (they meet ds = 0 in dq)
                const Place& a = ahead;
                if (a.j == 0 && !warp_wait(&bars->q_full[a.items & 1u], (a.items >> 1) & 1u, TO_MMA)) return false;
                if (!warp_wait(&bars->k_full[k_ring.slot], k_ring.parity, TO_MMA)) return false;
                uint8_t* op = k_smem + (size_t)k_ring.slot * OP;
                const int have = a.w.t.len - (a.w.t.way + a.j) * TILE;
                if (have < TILE) zero_rows(op, DB, have, lane);
                tc_fence_after();
                if (elect_one()) {
                    product(tmem, q_smem + (a.items & 1u) * OP, op);
                    mma_commit(smem_u32(&bars->s_full));
                    if (a.j + 1 == a.w.n) mma_commit(smem_u32(&bars->q_empty[a.items & 1u]));
                }
                __syncwarp();
                k_ring.next(KS);
                return true;
            };
            auto dps = [&](const Place& a) -> bool {
                if (a.j == 0 && !warp_wait(&bars->do_full, a.items & 1u, TO_MMA)) return false;
                if (!warp_wait(&bars->v_full[v_ring.slot], v_ring.parity, TO_MMA)) return false;
                tc_fence_after();
                if (elect_one()) {
                    product(tmem + 128, do_smem, v_smem + (size_t)v_ring.slot * OP);
                    mma_commit(smem_u32(&bars->dp_full));
                    mma_commit(smem_u32(&bars->v_empty[v_ring.slot]));
                    if (a.j + 1 == a.w.n) mma_commit(smem_u32(&bars->do_empty));
                }
                __syncwarp();
                v_ring.next(VS);
                return true;
            };
            if (walk.more) ok = scores() && dps(ahead);
            while (walk.more && ok) {
                const Place now = ahead;
                if (++ahead.j == ahead.w.n) {
                    ahead.j = 0; ++ahead.items;
                    walk.next();
                    if (walk.more) ahead.w = work_of(walk);
                }
                const bool more = walk.more, last = now.j + 1 == now.w.n;
                const uint64_t keys = make_smem_desc_mn_sw128(smem_u32(k_smem + (size_t)k_use.slot * OP), 16384);
                auto sum_keys = [&](uint32_t d, uint32_t a) {
#pragma unroll
                    for (int s = 0; s < 8; ++s) mma_f16_ts(d, a + quarter_column(s), keys + (uint64_t)(s * 128), idesc_q, now.j > 0 || s > 0);
                };
                if (!warp_wait(&bars->p_ready, tiles & 1u, TO_MMA)) { ok = false; break; }
                tc_fence_after();
                if (elect_one()) sum_keys(tmem + 384, tmem);
                __syncwarp();
                if (more && !scores()) { ok = false; break; }
                if (!warp_wait(&bars->ds_ready, tiles & 1u, TO_MMA)) { ok = false; break; }
                tc_fence_after();
                if (elect_one()) {
                    sum_keys(tmem + 256, tmem + 128);
                    mma_commit(smem_u32(&bars->k_empty[k_use.slot]));
                    if (last) mma_commit(smem_u32(&bars->dq_full));
                }
                __syncwarp();
                if (more && !dps(ahead)) { ok = false; break; }
                k_use.next(KS);
                ++tiles;
            }
            if (elect_one()) mma_commit(smem_u32(&bars->drain));
            __syncwarp();
            mbar_wait_quiet(smem_u32(&bars->drain), 0u);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        const int part = (warp >> 2) - 1, r = (warp & 3) * 32 + lane;      // which quarter of the columns
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_addr = tmem + lanes + part * 32, dp_addr = s_addr + 128;
        const int my_tok = r >> p.pack_shift, my_head = r & (p.pack - 1);
        const uint64_t scale2 = pair_of(p.scale_log2, p.scale_log2);
        uint32_t tiles = 0, items = 0;
        bool ok = true;
        // Statistics of an item's rows, eight to a warp: the lanes that share a row (8 or 16) read 16 bytes of out and of its gradient each (from L2, where
        // the producer has had them brought) before the epilogue of the item in front; behind it they are added up and put down.
        constexpr int LANES = 8 * DB, ROWS = 32 / LANES, PARTS = 8 / ROWS;
        const int sub = lane / LANES, c8 = (lane % LANES) * 8, stat_row = (warp - 4) * 8;
        uint4 o8[PARTS], d8[PARTS];
        float lse1 = 0.0f;
        auto row_of = [&](const Work& w, int row, int64_t& token, int& head) -> bool {
            const int a = w.t.at + (row >> p.pack_shift);
            token = w.t.t0 + a; head = w.head0 + (row & (p.pack - 1));
            return a < w.t.len;
        };
        auto fetch = [&](const Work& w) {
            int64_t token;
            int head;
            if (lane < 8 && row_of(w, stat_row + lane, token, head)) lse1 = p.lse[token * p.heads + head];
#pragma unroll
            for (int i = 0; i < PARTS; ++i) {
                o8[i] = d8[i] = make_uint4(0u, 0u, 0u, 0u);
                if (row_of(w, stat_row + i * ROWS + sub, token, head) && c8 < p.head_dim) {
                    o8[i] = __ldg(reinterpret_cast<const uint4*>(p.out + token * p.ld_out + (int64_t)head * p.head_dim + c8));
                    d8[i] = __ldg(reinterpret_cast<const uint4*>(p.dout + token * p.ld_dout + (int64_t)head * p.head_dim + c8));
                }
            }
        };
        auto put_down = [&](const Work& w) {
#pragma unroll
            for (int i = 0; i < PARTS; ++i) {
                float a[8], b[8], acc = 0.0f;
                unpack_bf16(o8[i], a);
                unpack_bf16(d8[i], b);
#pragma unroll
                for (int k = 0; k < 8; ++k) acc = fmaf(a[k], b[k], acc);
#pragma unroll
                for (int s = LANES / 2; s > 0; s >>= 1) acc += __shfl_xor_sync(0xFFFFFFFFu, acc, s);
                if (lane % LANES == 0) bars->delta[stat_row + i * ROWS + sub] = -acc;
            }
            __syncwarp();
            if (lane < 8) {
                int64_t token;
                int head;
                bars->lse[stat_row + lane] = row_of(w, stat_row + lane, token, head) ? -lse1 * LOG2E : 0.0f;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars->stat_full));
        };
        Walk walk(p.table, p.items, p.packs);
        Work w;
        bool more = walk.more;
        if (more) { w = work_of(walk); fetch(w); put_down(w); }
        for (; more && ok; ++items) {
            const int at = w.t.at + my_tok;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->stat_full), items & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
            if (!ok) break;
            const float off = bars->lse[r], delta = bars->delta[r];
            const uint64_t off2 = pair_of(off, off), delta2 = pair_of(delta, delta);
            uint64_t rho2[2] = {0, 0};
            for (int j = 0; j < w.n; ++j, ++tiles) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->s_full), tiles & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
                if (!ok) break;
                tc_fence_after();
                uint32_t s[2][16];
                uint64_t pr[16];
                tmem_ld_x16(s_addr, s[0]);
                tmem_wait_ld();
                tmem_ld_x16(s_addr + 16, s[1]);
                const int key0 = (w.t.way + j) * TILE;
                const bool masked = key0 + TILE - 1 > w.t.at;
                const int lim = at - key0 - part * 32;   // this row's last key among the 32
                auto hide = [&](uint64_t x, int k) {         // zeros behind it
                    float a, b;
                    split_pair(x, a, b);
                    return pair_of(2 * k > lim ? 0.0f : a, 2 * k + 1 > lim ? 0.0f : b);
                };
                auto form_p = [&](auto diagonal) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (h == 1) tmem_wait_ld();
                        uint32_t e[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            uint64_t& x = pr[h * 8 + k];
                            x = ex2_pair(fma2(pair_of(__uint_as_float(s[h][2 * k]), __uint_as_float(s[h][2 * k + 1])), scale2, off2));
                            if constexpr (diagonal.value) x = hide(x, h * 8 + k);
                            e[k] = pack_pair(x);
                        }
                        tmem_st_x8(s_addr + h * 8, e);       // over this quarter's own scores
                    }
                };
                if (masked) form_p(std::true_type{});
                else form_p(std::false_type{});
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars->p_ready));
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->dp_full), tiles & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
                if (!ok) break;
                tc_fence_after();
                tmem_ld_x16(dp_addr, s[0]);
                tmem_wait_ld();
                tmem_ld_x16(dp_addr + 16, s[1]);
                auto form_ds = [&](auto diagonal) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (h == 1) tmem_wait_ld();
                        uint32_t e[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            uint64_t ds = mul2(pr[h * 8 + k], add2(pair_of(__uint_as_float(s[h][2 * k]), __uint_as_float(s[h][2 * k + 1])), delta2));
                            if constexpr (diagonal.value) ds = hide(ds, h * 8 + k);      // (also where dp is not finite)
                            rho2[k & 1] = add2(rho2[k & 1], ds);
                            e[k] = pack_pair(ds);
                        }
                        tmem_st_x8(dp_addr + h * 8, e);
                    }
                };
                if (masked) form_ds(std::true_type{});
                else form_ds(std::false_type{});
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars->ds_ready));
            }
            if (!ok) break;
            walk.next();
            more = walk.more;
            Work next = w;
            if (more) { next = work_of(walk); fetch(next); }
            // rho of the row from its quarters, in the places of lse and delta, which everybody has read (the last tile's ds has arrived only when all had): the
            // third and fourth leave theirs, the first and second add those and leave the two sums
            float rho, low, high;
            split_pair(add2(rho2[0], rho2[1]), low, high);
            rho = low + high;
            float* place = (part & 1) ? bars->delta : bars->lse;
            auto meet = [&](uint64_t* bar) -> bool { return __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(bar), items & 1u, abort_flag, p.timeout_word, TO_EPILOGUE)); };
            auto here = [&](uint64_t* bar) {
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(bar));
            };
            ok = meet(&bars->dq_full);
            if (!ok) break;
            if (part >= 2) {
                place[r] = rho;
                here(&bars->rho_low);
            } else {
                ok = meet(&bars->rho_low);
                if (!ok) break;
                place[r] = rho + place[r];
                here(&bars->rho_sum);
            }
            ok = meet(&bars->rho_sum);
            if (!ok) break;
            rho = bars->lse[r] + bars->delta[r];
            here(&bars->rho_read);
            const bool split = p.chunk > 0 && loops(w.t) > p.chunk;      // there are other pieces of this tile
            const int64_t sums_row = (int64_t)item_of_round(walk.round - 1) * TILE + r;
            if (part == 0 && at < w.t.len) {
                if (split) p.stat[sums_row] = make_float2(rho, delta);
                else p.delta[(int64_t)(w.t.t0 + at) * p.heads + w.head0 + my_head] = delta - rho;      // (negated)
            }
            tc_fence_after();
            __nv_bfloat16* dst[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int rr = (warp & 3) * 32 + (lane & ~3) + k, a = w.t.at + (rr >> p.pack_shift);
                dst[k] = a < w.t.len ? p.dq + (int64_t)(w.t.t0 + a) * p.ld_dq + (int64_t)(w.head0 + (rr & (p.pack - 1))) * p.head_dim : nullptr;
            }
            if (split) {                                     // query_join_kernel does what follows
                if (part * 32 < p.head_dim) {
#pragma unroll 1
                    for (int h = 0; h < 2; ++h) put_sums(tmem + lanes + 256 + h * 128 + part * 32, p.part + (sums_row * 2 + h) * (DB * 64) + part * 32);
                }
            } else if (part * 32 < p.head_dim) {
                uint32_t o[32];
                float f[32];
                __syncwarp();
                tmem_ld_x32(tmem + lanes + 256 + part * 32, o);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 32; ++k) f[k] = __uint_as_float(o[k]);
                tmem_ld_x32(tmem + lanes + 384 + part * 32, o);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 32; ++k) f[k] = fmaf(-rho, __uint_as_float(o[k]), f[k]) * p.scale;
                store_rows32(f, part * 32, p.head_dim, lane, dst);
            }
            tc_fence_before();
            ok = meet(&bars->rho_read);                      // the statistics' places are free
            if (!ok) break;
            if (more) { put_down(next); w = next; }
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
    uint32_t items, kv_heads;
    int32_t chunk;                          // > 0: items are pieces of tiles, of so many tiles of queries; a tile of several leaves its sums here:
    float* part;                            // [item][row][dv, dk: 64 DB each]
    int32_t pack, pack_shift, group, heads, head_dim;
    float scale, scale_log2;
    unsigned int* timeout_word;
};

// A tile's dO is done with before its queries are, and is needed later: rings of their own.
template <int DB> struct KeyStages { static constexpr int Q = DB == 1 ? 4 : 3, D = DB == 1 ? 4 : 2; };
constexpr int LSE_STAGES = 2;               // (delta is needed half a tile later than lse: one place)

template <int DB>
struct __align__(16) KeyBars {
    float lse[LSE_STAGES][TILE], delta[TILE];      // of each query row, negated: lse times log2 e, delta
    uint64_t kv_full, kv_empty, q_full[KeyStages<DB>::Q], q_empty[KeyStages<DB>::Q], do_full[KeyStages<DB>::D], do_empty[KeyStages<DB>::D];
    uint64_t lse_full[LSE_STAGES], lse_empty[LSE_STAGES], delta_full, delta_empty, s_full, dp_full, p_ready, ds_ready, done, drain;
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
    constexpr uint32_t QS = KeyStages<DB>::Q, DS = KeyStages<DB>::D;
    uint8_t* q_smem = smem + 2 * OP;                         // queries
    uint8_t* do_smem = q_smem + QS * OP;                     // the gradient of their outputs
    KeyBars<DB>* bars = reinterpret_cast<KeyBars<DB>*>(do_smem + DS * OP);
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int tok = TILE >> p.pack_shift, passes = p.group >> p.pack_shift;

    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&bars->kv_full), 1); mbar_init(smem_u32(&bars->kv_empty), 1);
        for (uint32_t i = 0; i < QS; ++i) { mbar_init(smem_u32(&bars->q_full[i]), 1); mbar_init(smem_u32(&bars->q_empty[i]), 1); }
        for (uint32_t i = 0; i < DS; ++i) { mbar_init(smem_u32(&bars->do_full[i]), 1); mbar_init(smem_u32(&bars->do_empty[i]), 1); }
        for (int i = 0; i < LSE_STAGES; ++i) { mbar_init(smem_u32(&bars->lse_full[i]), 2); mbar_init(smem_u32(&bars->lse_empty[i]), 16); }
        mbar_init(smem_u32(&bars->delta_full), 2); mbar_init(smem_u32(&bars->delta_empty), 16);
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
    struct Work { AttnTile t; int kv, first, per, n, head0, i, left; };      // head0, i, left: where they begin (pieces: step t.way)
    auto work_of = [&](const Walk& k) {
        Work w;
        w.kv = (int)k.sub;
        w.t = k.tile;
        w.first = w.t.at >> (7 - p.pack_shift);
        w.per = ((w.t.len + tok - 1) >> (7 - p.pack_shift)) - w.first;
        w.n = w.per * passes;
        w.head0 = w.kv * p.group; w.i = w.first; w.left = w.per;
        if (p.chunk > 0) {
            const int j0 = w.t.way, pass = j0 / w.per, in = j0 - pass * w.per;
            w.n = min(p.chunk, w.n - j0);
            w.head0 += pass * p.pack; w.i += in; w.left -= in;
        }
        return w;
    };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 0) {
            Ring q_ring, do_ring;
            uint32_t tiles = 0, kv_uses = 0;
            bool ok = true;
            auto load = [&](const CUtensorMap* map, uint64_t* full_bar, uint8_t* dst_op, int head, int row) {
                if (elect_one()) {
                    const uint32_t full = smem_u32(full_bar), dst = smem_u32(dst_op);
                    mbar_arrive_expect_tx(full, OP);
#pragma unroll
                    for (int b = 0; b < DB; ++b) tma_load_3d(dst + b * 16384, map, full, b * 64, head, row);
                }
                __syncwarp();
            };
            for (Walk walk(p.table, p.items, p.kv_heads); walk.more && ok; walk.next()) {
                const Work w = work_of(walk);
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
                const uint32_t item = item_of_round(walk.round + 1);
                if (item < p.items) {                        // the next item's keys and values come out of L2
                    const AttnTile t = uniform_tile(walk.after);
                    const int kv = (int)(item - item / p.kv_heads * p.kv_heads);
                    if (elect_one()) {
#pragma unroll
                        for (int b = 0; b < DB; ++b) { tma_prefetch_3d(&tm_k, b * 64, kv, t.t0 + t.at); tma_prefetch_3d(&tm_v, b * 64, kv, t.t0 + t.at); }
                    }
                    __syncwarp();
                }
                int head0 = w.head0, i = w.i, left = w.left;
                for (int j = 0; j < w.n; ++j, ++tiles, q_ring.next(QS), do_ring.next(DS)) {
                    if (!warp_wait(&bars->q_empty[q_ring.slot], q_ring.parity ^ 1u, TO_PRODUCER)) { ok = false; break; }
                    load(&tm_q, &bars->q_full[q_ring.slot], q_smem + (size_t)q_ring.slot * OP, head0, w.t.t0 + i * tok);
                    if (!warp_wait(&bars->do_empty[do_ring.slot], do_ring.parity ^ 1u, TO_PRODUCER)) { ok = false; break; }
                    load(&tm_do, &bars->do_full[do_ring.slot], do_smem + (size_t)do_ring.slot * OP, head0, w.t.t0 + i * tok);
                    ++i;
                    if (--left == 0) { left = w.per; i = w.first; head0 += p.pack; }
                }
            }
            if (!ok) {
                for (uint32_t i = kv_uses > 1 ? kv_uses - 2 : 0u; i < kv_uses; ++i) mbar_wait_quiet(smem_u32(&bars->kv_full), i & 1u, 1u << 14);
                for (uint32_t i = tiles > QS ? tiles - QS : 0u; i <= tiles; ++i) mbar_wait_quiet(smem_u32(&bars->q_full[i % QS]), (i / QS) & 1u, 1u << 14);
                for (uint32_t i = tiles > DS ? tiles - DS : 0u; i < tiles; ++i) mbar_wait_quiet(smem_u32(&bars->do_full[i % DS]), (i / DS) & 1u, 1u << 14);
            }
        } else if (warp == 1) {
            const uint32_t n_d = (uint32_t)((p.head_dim + 15) / 16 * 16), steps = n_d / 16;
            const uint32_t idesc_s = make_idesc(1, 1, 1, 128, 128), idesc_g = make_idesc(1, 1, 1, 128, n_d) | IDESC_B_MN;
            Ring q_ring, do_ring;
            uint32_t kv_uses = 0, p_uses = 0, ds_uses = 0;
            bool ok = true;
            auto product = [&](uint32_t d, const uint8_t* a_op, const uint8_t* b_op) {
                const uint64_t a = make_smem_desc_sw128(smem_u32(a_op)), b = make_smem_desc_sw128(smem_u32(b_op));
#pragma unroll
                for (uint32_t k = 0; k < 4 * DB; ++k) {
                    const uint64_t off = (uint64_t)((k >> 2) * 1024 + (k & 3) * 2);
                    if (k < steps) mma_f16_ss(d, a + off, b + off, idesc_s, k > 0);
                }
            };
            auto gradient = [&](uint32_t d, uint32_t a, const uint8_t* b_op, bool more) {
                const uint64_t b = make_smem_desc_mn_sw128(smem_u32(b_op), 16384);
#pragma unroll
                for (int s = 0; s < 8; ++s) mma_f16_ts(d, a + quarter_column(s), b + (uint64_t)(s * 128), idesc_g, more || s > 0);
            };
            for (Walk walk(p.table, p.items, p.kv_heads); walk.more && ok; walk.next()) {
                const Work w = work_of(walk);
                if (!warp_wait(&bars->kv_full, kv_uses++ & 1u, TO_MMA)) { ok = false; break; }
                int i = w.i, left = w.left, have = TILE;   // have: query rows of the tile at `q_ring` that are there
                // The tile's queries (its dO) have arrived; rows behind the sequence's end become zeros in both operands (they meet P = dS = 0).
                auto q_arrived = [&](const Ring& at) -> bool {
                    if (!warp_wait(&bars->q_full[at.slot], at.parity, TO_MMA)) return false;
                    have = (w.t.len - i * tok) << p.pack_shift;
                    if (have < TILE) zero_rows(q_smem + (size_t)at.slot * OP, DB, have, lane);
                    ++i;
                    if (--left == 0) { left = w.per; i = w.first; }
                    tc_fence_after();
                    return true;
                };
                auto do_arrived = [&](const Ring& at) -> bool {      // (of the same tile, behind its queries)
                    if (!warp_wait(&bars->do_full[at.slot], at.parity, TO_MMA)) return false;
                    if (have < TILE) zero_rows(do_smem + (size_t)at.slot * OP, DB, have, lane);
                    tc_fence_after();
                    return true;
                };
                if (!q_arrived(q_ring) || !do_arrived(do_ring)) { ok = false; break; }
                if (elect_one()) {
                    product(tmem, kv_smem, q_smem + (size_t)q_ring.slot * OP);
                    mma_commit(smem_u32(&bars->s_full));
                    product(tmem + 128, kv_smem + OP, do_smem + (size_t)do_ring.slot * OP);
                    mma_commit(smem_u32(&bars->dp_full));
                    if (w.n == 1) mma_commit(smem_u32(&bars->kv_empty));
                }
                __syncwarp();
                for (int j = 0; j < w.n && ok; ++j) {
                    Ring q_next = q_ring, do_next = do_ring;
                    q_next.next(QS); do_next.next(DS);
                    const bool more = j + 1 < w.n;
                    if (more && !q_arrived(q_next)) { ok = false; break; }
                    if (!warp_wait(&bars->p_ready, p_uses++ & 1u, TO_MMA)) { ok = false; break; }
                    tc_fence_after();
                    if (elect_one()) {
                        gradient(tmem + 256, tmem, do_smem + (size_t)do_ring.slot * OP, j > 0);
                        mma_commit(smem_u32(&bars->do_empty[do_ring.slot]));
                        if (more) {
                            product(tmem, kv_smem, q_smem + (size_t)q_next.slot * OP);
                            mma_commit(smem_u32(&bars->s_full));
                        }
                    }
                    __syncwarp();
                    if (more && !do_arrived(do_next)) { ok = false; break; }
                    if (!warp_wait(&bars->ds_ready, ds_uses++ & 1u, TO_MMA)) { ok = false; break; }
                    tc_fence_after();
                    if (elect_one()) {
                        gradient(tmem + 384, tmem + 128, q_smem + (size_t)q_ring.slot * OP, j > 0);
                        mma_commit(smem_u32(&bars->q_empty[q_ring.slot]));
                        if (more) {
                            product(tmem + 128, kv_smem + OP, do_smem + (size_t)do_next.slot * OP);
                            mma_commit(smem_u32(&bars->dp_full));
                            if (j + 2 == w.n) mma_commit(smem_u32(&bars->kv_empty));
                        } else {
                            mma_commit(smem_u32(&bars->done));
                        }
                    }
                    __syncwarp();
                    q_ring = q_next; do_ring = do_next;
                }
            }
            if (elect_one()) mma_commit(smem_u32(&bars->drain));
            __syncwarp();
            mbar_wait_quiet(smem_u32(&bars->drain), 0u);
        } else {
            Ring ring;
            uint32_t tiles = 0;
            bool ok = true;
            for (Walk walk(p.table, p.items, p.kv_heads); walk.more && ok; walk.next()) {
                const Work w = work_of(walk);
                int head0 = w.head0, i = w.i, left = w.left;
                for (int j = 0; j < w.n; ++j, ++tiles, ring.next(LSE_STAGES)) {
                    float lse[2], delta[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {            // rows behind the end: P = e^(0 - infinity) = 0, dS = 0
                        const int r = (warp - 2) * 64 + h * 32 + lane, at = i * tok + (r >> p.pack_shift);
                        lse[h] = -INFINITY; delta[h] = 0.0f;
                        if (at < w.t.len) {
                            const int64_t row = (int64_t)(w.t.t0 + at) * p.heads + head0 + (r & (p.pack - 1));
                            lse[h] = -p.lse[row] * LOG2E; delta[h] = p.delta[row];
                        }
                    }
                    if (!warp_wait(&bars->lse_empty[ring.slot], ring.parity ^ 1u, TO_PRODUCER)) { ok = false; break; }
#pragma unroll
                    for (int h = 0; h < 2; ++h) bars->lse[ring.slot][(warp - 2) * 64 + h * 32 + lane] = lse[h];
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&bars->lse_full[ring.slot]));
                    if (!warp_wait(&bars->delta_empty, (tiles & 1u) ^ 1u, TO_PRODUCER)) { ok = false; break; }
#pragma unroll
                    for (int h = 0; h < 2; ++h) bars->delta[(warp - 2) * 64 + h * 32 + lane] = delta[h];
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&bars->delta_full));
                    ++i;
                    if (--left == 0) { left = w.per; i = w.first; head0 += p.pack; }
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        const int part = (warp >> 2) - 1, r = (warp & 3) * 32 + lane;      // which quarter of the columns
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_addr = tmem + lanes + part * 32, dp_addr = s_addr + 128;
        const uint64_t scale2 = pair_of(p.scale_log2, p.scale_log2);
        uint32_t uses = 0, done_uses = 0;
        Ring ring;
        bool ok = true;
        for (Walk walk(p.table, p.items, p.kv_heads); walk.more && ok; walk.next()) {
            const Work w = work_of(walk);
            const int key = w.t.at + r;
            int i = w.i, left = w.left;
            for (int j = 0; j < w.n; ++j, ++uses, ring.next(LSE_STAGES)) {
                // column c of this quarter is query row part * 32 + c: token i * tok + (part * 32 + c) / pack; it sees this row's key from `from` on
                const bool masked = i * tok < w.t.at + TILE - 1;
                const int from = (key - i * tok) * p.pack - part * 32;
                ++i;
                if (--left == 0) { left = w.per; i = w.first; }
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->lse_full[ring.slot]), ring.parity, abort_flag, p.timeout_word, TO_EPILOGUE));
                if (!ok) break;
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->s_full), uses & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
                if (!ok) break;
                tc_fence_after();
                uint32_t s[2][16];
                uint64_t pr[16];
                tmem_ld_x16(s_addr, s[0]);
                const float4* lse = reinterpret_cast<const float4*>(&bars->lse[ring.slot][part * 32]);      // negated, like delta
                const float4* delta = reinterpret_cast<const float4*>(&bars->delta[part * 32]);
                tmem_wait_ld();
                tmem_ld_x16(s_addr + 16, s[1]);
                auto form_p = [&](auto diagonal) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (h == 1) tmem_wait_ld();
                        uint32_t e[8];
#pragma unroll
                        for (int k = 0; k < 8; k += 2) {
                            const float4 l = lse[(h * 8 + k) / 2];
                            pr[h * 8 + k] = ex2_pair(fma2(pair_of(__uint_as_float(s[h][2 * k]), __uint_as_float(s[h][2 * k + 1])), scale2, pair_of(l.x, l.y)));
                            pr[h * 8 + k + 1] = ex2_pair(fma2(pair_of(__uint_as_float(s[h][2 * k + 2]), __uint_as_float(s[h][2 * k + 3])), scale2, pair_of(l.z, l.w)));
                        }
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            if constexpr (diagonal.value) {
                                float a, b;
                                split_pair(pr[h * 8 + k], a, b);
                                pr[h * 8 + k] = pair_of(h * 16 + 2 * k < from ? 0.0f : a, h * 16 + 2 * k + 1 < from ? 0.0f : b);
                            }
                            e[k] = pack_pair(pr[h * 8 + k]);
                        }
                        tmem_st_x8(s_addr + h * 8, e);           // over this quarter's own scores
                    }
                };
                if (masked) form_p(std::true_type{});
                else form_p(std::false_type{});
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) { mbar_arrive(smem_u32(&bars->p_ready)); mbar_arrive(smem_u32(&bars->lse_empty[ring.slot])); }
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->delta_full), uses & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
                if (!ok) break;
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->dp_full), uses & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
                if (!ok) break;
                tc_fence_after();
                tmem_ld_x16(dp_addr, s[0]);
                tmem_wait_ld();
                tmem_ld_x16(dp_addr + 16, s[1]);
                auto form_ds = [&](auto diagonal) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (h == 1) tmem_wait_ld();
                        uint32_t e[8];
#pragma unroll
                        for (int k = 0; k < 8; k += 2) {
                            const float4 d = delta[(h * 8 + k) / 2];
                            uint64_t a2 = mul2(pr[h * 8 + k], add2(pair_of(__uint_as_float(s[h][2 * k]), __uint_as_float(s[h][2 * k + 1])), pair_of(d.x, d.y)));
                            uint64_t b2 = mul2(pr[h * 8 + k + 1], add2(pair_of(__uint_as_float(s[h][2 * k + 2]), __uint_as_float(s[h][2 * k + 3])), pair_of(d.z, d.w)));
                            if constexpr (diagonal.value) {
                                float a, b;
                                split_pair(a2, a, b);
                                a2 = pair_of(h * 16 + 2 * k < from ? 0.0f : a, h * 16 + 2 * k + 1 < from ? 0.0f : b);
                                split_pair(b2, a, b);
                                b2 = pair_of(h * 16 + 2 * k + 2 < from ? 0.0f : a, h * 16 + 2 * k + 3 < from ? 0.0f : b);
                            }
                            e[k] = pack_pair(a2); e[k + 1] = pack_pair(b2);
                        }
                        tmem_st_x8(dp_addr + h * 8, e);
                    }
                };
                if (masked) form_ds(std::true_type{});
                else form_ds(std::false_type{});
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) { mbar_arrive(smem_u32(&bars->ds_ready)); mbar_arrive(smem_u32(&bars->delta_empty)); }
            }
            if (!ok) break;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->done), done_uses++ & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
            if (!ok) break;
            tc_fence_after();
            // two groups of warps have dv, two dk: every other 32 columns each
            const bool is_k = part >= 2;
            if (p.chunk > 0 && w.per * passes > p.chunk) {   // (other pieces of this tile) key_join_kernel does what follows
#pragma unroll 1
                for (int c = (part & 1) * 32; c < p.head_dim; c += 64)
                    put_sums(tmem + lanes + 256 + (is_k ? 128 : 0) + c, p.part + (((int64_t)walk.item * TILE + r) * 2 + (is_k ? 1 : 0)) * (DB * 64) + c);
                tc_fence_before();
                continue;
            }
            __nv_bfloat16* base = is_k ? p.dk : p.dv;
            const int64_t ld = is_k ? p.ld_dk : p.ld_dv;
            const float by = is_k ? p.scale : 1.0f;
            const int row0 = w.t.at + (warp & 3) * 32 + (lane & ~3);
            __nv_bfloat16* dst[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) dst[k] = row0 + k < w.t.len ? base + (int64_t)(w.t.t0 + row0 + k) * ld + (int64_t)w.kv * p.head_dim : nullptr;
#pragma unroll 1
            for (int c = (part & 1) * 32; c < p.head_dim; c += 64) {
                uint32_t o[32];
                float f[32];
                __syncwarp();
                tmem_ld_x32(tmem + lanes + 256 + (is_k ? 128 : 0) + c, o);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 32; ++k) f[k] = __uint_as_float(o[k]) * by;
                store_rows32(f, c, p.head_dim, lane, dst);
            }
            tc_fence_before();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, 512); }
}

// The pieces of a tile, added up in their order. A warp has a row, a lane four columns of it; block (piece, head or pack of heads, eighth of the rows), that
// of a tile's first piece does the tile.
template <int DB>
__global__ void __launch_bounds__(128) query_join_kernel(const __grid_constant__ QueryParams p)
{
    ahead_wait();
    ahead_release();
    const AttnTile t = p.table.few[blockIdx.x];
    const int tok = TILE >> p.pack_shift, pieces = ((min(t.at + tok, t.len) + TILE - 1) / TILE + p.chunk - 1) / p.chunk;
    if (t.way != 0 || pieces == 1) return;
    const int c = (threadIdx.x & 31) * 4;
    for (int i = 0; i < 4; ++i) {
        const int r = blockIdx.z * 16 + (threadIdx.x >> 5) * 4 + i, at = t.at + (r >> p.pack_shift), head = (int)blockIdx.y * p.pack + (r & (p.pack - 1));
        if (at >= t.len) break;
        float rho = 0.0f, delta = 0.0f, dq[4] = {0.0f, 0.0f, 0.0f, 0.0f}, kbar[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < pieces; ++s) {
            const int64_t row = ((int64_t)(blockIdx.x + s) * p.packs + blockIdx.y) * TILE + r;
            const float2 st = p.stat[row];
            rho += st.x; delta = st.y;
            if (c < p.head_dim) {
                const float4 a = *reinterpret_cast<const float4*>(p.part + row * 2 * (DB * 64) + c), b = *reinterpret_cast<const float4*>(p.part + (row * 2 + 1) * (DB * 64) + c);
                dq[0] += a.x; dq[1] += a.y; dq[2] += a.z; dq[3] += a.w;
                kbar[0] += b.x; kbar[1] += b.y; kbar[2] += b.z; kbar[3] += b.w;
            }
        }
        if (c == 0) p.delta[(int64_t)(t.t0 + at) * p.heads + head] = delta - rho;
        if (c < p.head_dim) {
            float f[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) f[k] = fmaf(-rho, kbar[k], dq[k]) * p.scale;
            *reinterpret_cast<uint2*>(p.dq + (int64_t)(t.t0 + at) * p.ld_dq + (int64_t)head * p.head_dim + c) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
        }
    }
}

template <int DB>
__global__ void __launch_bounds__(128) key_join_kernel(const __grid_constant__ KeyParams p)
{
    ahead_wait();
    ahead_release();
    const AttnTile t = p.table.few[blockIdx.x];
    const int tok = TILE >> p.pack_shift, per = ((t.len + tok - 1) >> (7 - p.pack_shift)) - (t.at >> (7 - p.pack_shift));
    const int pieces = (per * (p.group >> p.pack_shift) + p.chunk - 1) / p.chunk;
    if (t.way != 0 || pieces == 1) return;
    const int c = (threadIdx.x & 31) * 4;
    if (c >= p.head_dim) return;
    for (int i = 0; i < 4; ++i) {
        const int r = blockIdx.z * 16 + (threadIdx.x >> 5) * 4 + i;
        if (t.at + r >= t.len) break;
        float dv[4] = {0.0f, 0.0f, 0.0f, 0.0f}, dk[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < pieces; ++s) {
            const int64_t row = ((int64_t)(blockIdx.x + s) * p.kv_heads + blockIdx.y) * TILE + r;
            const float4 a = *reinterpret_cast<const float4*>(p.part + row * 2 * (DB * 64) + c), b = *reinterpret_cast<const float4*>(p.part + (row * 2 + 1) * (DB * 64) + c);
            dv[0] += a.x; dv[1] += a.y; dv[2] += a.z; dv[3] += a.w;
            dk[0] += b.x; dk[1] += b.y; dk[2] += b.z; dk[3] += b.w;
        }
        const int64_t token = t.t0 + t.at + r, col = (int64_t)blockIdx.y * p.head_dim + c;
        *reinterpret_cast<uint2*>(p.dv + token * p.ld_dv + col) = make_uint2(pack_bf16(dv[0], dv[1]), pack_bf16(dv[2], dv[3]));
        *reinterpret_cast<uint2*>(p.dk + token * p.ld_dk + col) = make_uint2(pack_bf16(dk[0] * p.scale, dk[1] * p.scale), pack_bf16(dk[2] * p.scale, dk[3] * p.scale));
    }
}

template <int DB>
qless_status launch_backward(const CUtensorMap& q, const CUtensorMap& d, const CUtensorMap& k, const CUtensorMap& v, const CUtensorMap& o, const QueryParams& qp, const KeyParams& kp, cudaStream_t st)
{
    const size_t op = (size_t)DB * 16384;
    const size_t q_smem = 1024 + (3 + QueryStages<DB>::K + QueryStages<DB>::V) * op + sizeof(QueryBars<DB>), k_smem = 1024 + (2 + KeyStages<DB>::Q + KeyStages<DB>::D) * op + sizeof(KeyBars<DB>);
    static_assert(1024 + (3 + QueryStages<DB>::K + QueryStages<DB>::V) * DB * 16384 + sizeof(QueryBars<DB>) <= 227 * 1024 &&
                  1024 + (2 + KeyStages<DB>::Q + KeyStages<DB>::D) * DB * 16384 + sizeof(KeyBars<DB>) <= 227 * 1024, "shared memory of an SM");
    { ProfileScope ps("attention_dq", st);
      QLESS_CUDA_TRY((allow_full_smem<attention_dq_kernel<DB>>()));
      QLESS_CUDA_TRY(launch_ahead(attention_dq_kernel<DB>, dim3((unsigned)std::min<int64_t>(qp.items, sm_count())), dim3(NTHREADS), q_smem, st, q, d, k, v, o, qp));
      if (qp.chunk > 0) { QLESS_CUDA_TRY(launch_ahead(query_join_kernel<DB>, dim3((unsigned)qp.table.tiles, qp.packs, 8), dim3(128), 0, st, qp)); count_launches(1); } }
    count_launches(1);
    { ProfileScope ps("attention_dkv", st);
      QLESS_CUDA_TRY((allow_full_smem<attention_dkv_kernel<DB>>()));
      QLESS_CUDA_TRY(launch_ahead(attention_dkv_kernel<DB>, dim3((unsigned)std::min<int64_t>(kp.items, sm_count())), dim3(NTHREADS), k_smem, st, q, d, k, v, kp));
      if (kp.chunk > 0) { QLESS_CUDA_TRY(launch_ahead(key_join_kernel<DB>, dim3((unsigned)kp.table.tiles, kp.kv_heads, 8), dim3(128), 0, st, kp)); count_launches(1); } }
    count_launches(1);
    return QLESS_OK;
}

}  // namespace

size_t attention_workspace(int64_t tokens, int64_t n, int32_t heads, int32_t kv_heads, bool backward)
{
    const int64_t tok = TILE / attn_pack(heads, kv_heads);
    size_t total = tiles_bytes(tokens, n, tok);
    total += split_bytes(tokens, heads, kv_heads, backward);
    if (backward) total += tiles_bytes(tokens, n, TILE) + align_up((size_t)tokens * heads * 4, 256);
    return total;
}

qless_status launch_attention_backward(const AttnArgs& a, uint8_t* ws, unsigned int* timeout_word, cudaStream_t st)
{
    const int32_t pack = attn_pack(a.heads, a.kv_heads), tok = TILE / pack, packs = a.heads / pack;
    std::vector<AttnTile> queries = query_tiles(a, tok), keys = key_tiles(a);
    if (queries.empty()) return QLESS_OK;
    // (fewer key tiles than query tiles, and no more key heads than packs)
    QLESS_REQUIRE((int64_t)queries.size() * packs < MOST_ITEMS - 65536, QLESS_ERR_UNSUPPORTED, "too many tiles: %zu of %d heads", queries.size(), packs);
    int32_t shift = 0;
    while ((1 << shift) < pack) ++shift;
    AttnTile* q_list = reinterpret_cast<AttnTile*>(ws);
    AttnTile* k_list = reinterpret_cast<AttnTile*>(ws + tiles_bytes(a.tokens, a.n, tok));
    float* delta = reinterpret_cast<float*>(ws + tiles_bytes(a.tokens, a.n, tok) + tiles_bytes(a.tokens, a.n, TILE));
    QueryParams qp;
    KeyParams kp;
    const int32_t passes = a.heads / a.kv_heads / pack;
    qp.chunk = split_tiles(&queries, packs, SPLIT_BACKWARD, [&](const AttnTile& t) { return (std::min(t.at + tok, t.len) + TILE - 1) / TILE; });
    kp.chunk = split_tiles(&keys, a.kv_heads, SPLIT_BACKWARD, [&](const AttnTile& t) { return ((t.len + tok - 1) / tok - t.at / tok) * passes; });
    // (one room for both: the keys' kernel begins when the queries' sums are joined)
    uint8_t* room = reinterpret_cast<uint8_t*>(delta) + align_up((size_t)a.tokens * a.heads * 4, 256);
    qp.stat = reinterpret_cast<float2*>(room); qp.part = kp.part = reinterpret_cast<float*>(room + (size_t)SPLIT_ROUNDS * sm_count() * TILE * sizeof(float2));
    qless_status s;
    if ((s = put_table(queries, &qp.table, q_list, st)) != QLESS_OK) return s;
    if ((s = put_table(keys, &kp.table, k_list, st)) != QLESS_OK) return s;
    CUtensorMap q, d, k, v, o;
    if ((s = head_map(&q, a.q, a.ld_q, a.heads, a.head_dim, a.tokens, pack, tok)) != QLESS_OK) return s;
    if ((s = head_map(&d, a.dout, a.ld_dout, a.heads, a.head_dim, a.tokens, pack, tok)) != QLESS_OK) return s;
    if ((s = head_map(&o, a.out_in, a.ld_out, a.heads, a.head_dim, a.tokens, pack, tok)) != QLESS_OK) return s;
    if ((s = head_map(&k, a.k, a.ld_k, a.kv_heads, a.head_dim, a.tokens, 1, TILE)) != QLESS_OK) return s;
    if ((s = head_map(&v, a.v, a.ld_v, a.kv_heads, a.head_dim, a.tokens, 1, TILE)) != QLESS_OK) return s;
    qp.out = reinterpret_cast<const __nv_bfloat16*>(a.out_in); qp.dout = reinterpret_cast<const __nv_bfloat16*>(a.dout); qp.lse = a.lse_in; qp.delta = delta;
    qp.dq = reinterpret_cast<__nv_bfloat16*>(a.dq); qp.ld_out = a.ld_out; qp.ld_dout = a.ld_dout; qp.ld_dq = a.ld_dq;
    qp.packs = packs; qp.pack = pack; qp.pack_shift = shift; qp.group = a.heads / a.kv_heads; qp.heads = a.heads; qp.head_dim = a.head_dim;
    qp.items = (uint32_t)(queries.size() * packs); qp.scale = a.scale; qp.scale_log2 = a.scale * LOG2E; qp.timeout_word = timeout_word;
    kp.lse = a.lse_in; kp.delta = delta; kp.dk = reinterpret_cast<__nv_bfloat16*>(a.dk); kp.dv = reinterpret_cast<__nv_bfloat16*>(a.dv);
    kp.ld_dk = a.ld_dk; kp.ld_dv = a.ld_dv; kp.kv_heads = a.kv_heads; kp.pack = pack; kp.pack_shift = shift; kp.group = qp.group; kp.heads = a.heads; kp.head_dim = a.head_dim;
    kp.items = (uint32_t)(keys.size() * a.kv_heads); kp.scale = a.scale; kp.scale_log2 = qp.scale_log2; kp.timeout_word = timeout_word;
    return a.head_dim <= 64 ? launch_backward<1>(q, d, k, v, o, qp, kp, st) : launch_backward<2>(q, d, k, v, o, qp, kp, st);
}

}  // namespace qless
