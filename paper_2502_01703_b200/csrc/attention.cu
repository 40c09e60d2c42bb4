// Causal attention over packed sequences with grouped heads: the forward kernel, and the tables of work.
//
//   s_ij = scale <q_i, k_j> for j <= i in the same sequence,  m_i = max_j s_ij,  o_i = sum_j e^(s_ij - m_i) v_j / sum_j e^(s_ij - m_i),
//   lse_i = m_i + log sum_j e^(s_ij - m_i)
//
// One pass over the keys per tile of queries; scores never leave the SM. A block works on two tiles of 128 query rows that share the copies of
// keys and values: while one tile's eight warps take exponentials, the tensor core works on the other's products.
//   warp 0        TMA: queries of a tile once, keys and values through a ring of tiles
//   warp 1        tcgen05: S = Q K^T (both from shared memory), O += P V (P from tensor memory, V as rows of tokens)
//   warps 4-11    tile 0: two threads share a row, half of the keys each: maximum, exponentials in fp32, P rounded to bf16 over S in tensor memory
//   warps 12-19   tile 1
// Tensor memory: S (or P) and O of both tiles, 4 x 128 columns. Running maximum: O and the sum are rescaled only when the maximum has grown by
// more than 2^8 since the reference was taken (e^(s - r) then stays below 2^8: neither fp32 sums nor bf16's relative rounding mind).
// P is rounded to bf16 (at most 2^-8 of each probability, independent of each other; the sum is that of the unrounded ones), O and the sums are fp32.
// Bound: 128 x 128 exponentials take the special-function units 1024 clocks, the two products of the same tile (head_dim 128) 1024 of the tensor core; what is
// measured for a pair of tiles is 3.5 to 3.8 thousand clocks, of which a tile's own chain (scores, maxima, exponentials, its products) takes nearly all: two
// 128-column tiles with their sums fill tensor memory, so the next scores of a tile wait for its P to be read. Two examples of 16383 tokens in all (32/8 heads of
// 128): 1.05 ms as a single call (1.11 PFLOP/s), 1.2 ms in a long row of them (0.97); short examples pay for the first loads and the epilogue of their items.
// Some of the exponentials on the fp32 units instead (a polynomial; from one pair in two to one in eight): no difference beyond 1 %.
// One thread to a row (four warps to a tile): 170 us instead of 141 for 32 examples of 16381 tokens in all, the same for long documents.
#include <algorithm>
#include <string.h>

#include "attention_common.cuh"

namespace qless {

namespace attn {

namespace {

constexpr int NTHREADS = 640, MAX_STAGES = 10;
constexpr float SLACK = 8.0f;               // powers of two that the maximum may grow before O is rescaled

struct ForwardParams {
    TileTable table;
    __nv_bfloat16* out; float* lse;
    int64_t ld_out;
    uint32_t items, packs;                  // packs: heads / pack
    int32_t chunk;                          // > 0: items are pieces of tiles, of so many tiles of keys; a tile of several leaves its sums here:
    float* part; float2* stat;              // [item][row][64 DB]: O before its division; [item][row]: reference, sum
    int32_t pack, pack_shift, group, heads, head_dim, stages;
    float scale_log2;
    unsigned int* timeout_word;
};

struct __align__(8) Bars {
    uint64_t q_full[2], q_empty[2], full[MAX_STAGES], empty[MAX_STAGES], s_full[2], p_ready[2][2], o_full[2], drain;      // P in two halves of the keys
    uint64_t met[2][4];                     // the two warps of 32 rows have put down what the other needs
    float swap[2][2][2][TILE];              // [turn][tile][half of the keys]: maxima, and sums at the end
    uint32_t tmem_base, abort_flag;
};

// DB: 64-column blocks of a head (head_dim up to 64 or 128).
template <int DB>
__global__ void __launch_bounds__(NTHREADS, 1)
attention_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                 const __grid_constant__ ForwardParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    constexpr int OP = DB * 16384;                           // bytes of a 128-row operand
    uint8_t* q_smem = smem;
    uint8_t* ring_smem = smem + 2 * OP;
    const uint32_t nS = (uint32_t)p.stages;
    Bars* bars = reinterpret_cast<Bars*>(ring_smem + (size_t)nS * OP);
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int tok = TILE >> p.pack_shift;                           // tokens of a 128-row tile

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bars->q_full[i]), 1); mbar_init(smem_u32(&bars->q_empty[i]), 1);
            mbar_init(smem_u32(&bars->s_full[i]), 1); mbar_init(smem_u32(&bars->p_ready[i][0]), 8); mbar_init(smem_u32(&bars->p_ready[i][1]), 4);
            for (int k = 0; k < 4; ++k) mbar_init(smem_u32(&bars->met[i][k]), 2);
            mbar_init(smem_u32(&bars->o_full[i]), 1);
        }
        for (uint32_t i = 0; i < MAX_STAGES; ++i) { mbar_init(smem_u32(&bars->full[i]), 1); mbar_init(smem_u32(&bars->empty[i]), 1); }
        mbar_init(smem_u32(&bars->drain), 1);
        bars->abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tm_q); prefetch_tmap(&tm_k); prefetch_tmap(&tm_v);
    }
    if (warp == 1) { tmem_alloc(smem_u32(&bars->tmem_base), 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;                   // S (P) of tile i at 128 i, O at 256 + 128 i
    ahead_wait();
    ahead_release();

    auto warp_wait = [&](uint64_t* bar, uint32_t parity, uint32_t code) -> bool {
        const bool w = mbar_wait(smem_u32(bar), parity, abort_flag, p.timeout_word, code);
        return __all_sync(0xFFFFFFFFu, w);
    };
    // item -> tile, first head, key head; loops of the two row tiles over the keys (0: the second one does not exist)
    struct Work { AttnTile t; int head0, kv, j0, n[2]; bool split; };      // j0: first tile of keys; split: there are other pieces
    auto work_of = [&](const Walk& k) {
        Work w;
        w.t = k.tile;
        w.head0 = (int)k.sub * p.pack; w.kv = w.head0 / p.group;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int first = w.t.at + x * tok;
            w.n[x] = first < w.t.len && (x == 0 || w.t.way == 0) ? (min(first + tok, w.t.len) + TILE - 1) / TILE : 0;
        }
        w.j0 = w.t.way >> 1; w.split = false;
        if (p.chunk > 0) { w.split = w.n[0] > p.chunk; w.n[0] = min(p.chunk, w.n[0] - w.j0); }
        return w;
    };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 0) {
            Ring ring;
            uint32_t it = 0, q_uses[2] = {0, 0};
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
            for (Walk walk(p.table, p.items, p.packs); walk.more && ok; walk.next()) {
                const Work w = work_of(walk);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (w.n[x] == 0 || !ok) continue;
                    if (!warp_wait(&bars->q_empty[x], (q_uses[x] & 1u) ^ 1u, TO_PRODUCER)) { ok = false; break; }
                    ++q_uses[x];
                    if (elect_one()) {
                        const uint32_t full = smem_u32(&bars->q_full[x]), dst = smem_u32(q_smem + x * OP);
                        mbar_arrive_expect_tx(full, OP);
#pragma unroll
                        for (int b = 0; b < DB; ++b) tma_load_3d(dst + b * 16384, &tm_q, full, b * 64, w.head0, w.t.t0 + w.t.at + x * tok);
                    }
                    __syncwarp();
                    if (x == 0) load(&tm_k, w.kv, w.t.t0 + w.j0 * TILE);
                }
                if (ok) load(&tm_v, w.kv, w.t.t0 + w.j0 * TILE);
                const uint32_t item = item_of_round(walk.round + 1);
                if (item < p.items) {                        // the next item's queries come out of L2
                    const AttnTile t = uniform_tile(walk.after);
                    const int head0 = (int)(item - item / p.packs * p.packs) * p.pack;
                    if (elect_one()) {
#pragma unroll
                        for (int b = 0; b < DB; ++b) {
                            tma_prefetch_3d(&tm_q, b * 64, head0, t.t0 + t.at);
                            if (t.way == 0 && t.at + tok < t.len) tma_prefetch_3d(&tm_q, b * 64, head0, t.t0 + t.at + tok);
                        }
                    }
                    __syncwarp();
                }
                const int n = max(w.n[0], w.n[1]);
                for (int j = 1; j < n && ok; ++j) {
                    load(&tm_k, w.kv, w.t.t0 + (w.j0 + j) * TILE);
                    if (ok) load(&tm_v, w.kv, w.t.t0 + (w.j0 + j) * TILE);
                }
            }
            // nothing of this block's copies is in flight when it leaves (the other roles wait for all of them unless one gave up)
            if (!ok)
                for (uint32_t j = it > nS ? it - nS : 0u; j < it; ++j)
                    if (!mbar_wait_quiet(smem_u32(&bars->full[j % nS]), (j / nS) & 1u, 1u << 14)) break;
        } else if (warp == 1) {
            const uint32_t n_pv = (uint32_t)((p.head_dim + 15) / 16 * 16), steps = n_pv / 16;      // columns of a head that are there
            const uint32_t idesc_s = make_idesc(1, 1, 1, 128, 128), idesc_o = make_idesc(1, 1, 1, 128, n_pv) | IDESC_B_MN;
            Ring ring;
            uint32_t q_uses[2] = {0, 0}, p_uses[2] = {0, 0};
            bool ok = true;
            auto scores = [&](int x, const uint8_t* k_op) {
                if (elect_one()) {
                    const uint64_t a = make_smem_desc_sw128(smem_u32(q_smem + x * OP)), b = make_smem_desc_sw128(smem_u32(k_op));
#pragma unroll
                    for (uint32_t k = 0; k < 4 * DB; ++k) {
                        const uint64_t off = (uint64_t)((k >> 2) * 1024 + (k & 3) * 2);
                        if (k < steps) mma_f16_ss(tmem + x * 128, a + off, b + off, idesc_s, k > 0);
                    }
                    mma_commit(smem_u32(&bars->s_full[x]));
                }
                __syncwarp();
            };
            for (Walk walk(p.table, p.items, p.packs); walk.more && ok; walk.next()) {
                const Work w = work_of(walk);
                const int n = max(w.n[0], w.n[1]);
                if (!warp_wait(&bars->full[ring.slot], ring.parity, TO_MMA)) { ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (w.n[x] == 0) continue;
                    if (!warp_wait(&bars->q_full[x], q_uses[x]++ & 1u, TO_MMA)) { ok = false; break; }
                    tc_fence_after();
                    scores(x, ring_smem + (size_t)ring.slot * OP);
                    if (w.n[x] == 1 && elect_one()) mma_commit(smem_u32(&bars->q_empty[x]));
                    __syncwarp();
                }
                if (!ok) break;
                if (elect_one()) mma_commit(smem_u32(&bars->empty[ring.slot]));
                __syncwarp();
                ring.next(nS);
                for (int j = 0; j < n && ok; ++j) {
                    const Ring v = ring;
                    ring.next(nS);
                    const Ring k = ring;
                    if (j + 1 < n) ring.next(nS);
                    uint8_t* v_op = ring_smem + (size_t)v.slot * OP;
                    if (!warp_wait(&bars->full[v.slot], v.parity, TO_MMA)) { ok = false; break; }
                    if (w.t.len - (w.j0 + j) * TILE < TILE) zero_rows(v_op, DB, w.t.len - (w.j0 + j) * TILE, lane);
                    if (j + 1 < n && !warp_wait(&bars->full[k.slot], k.parity, TO_MMA)) { ok = false; break; }
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if (j >= w.n[x]) continue;
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            if (!warp_wait(&bars->p_ready[x][half], p_uses[x] & 1u, TO_MMA)) { ok = false; break; }
                            tc_fence_after();
                            if (elect_one()) {
                                const uint64_t b = make_smem_desc_mn_sw128(smem_u32(v_op), 16384);
#pragma unroll
                                for (int s = half * 4; s < half * 4 + 4; ++s) mma_f16_ts(tmem + 256 + x * 128, tmem + x * 128 + half * 64 + (s & 3) * 8, b + (uint64_t)(s * 128), idesc_o, j > 0 || s > 0);
                                if (half == 1 && j + 1 == w.n[x]) mma_commit(smem_u32(&bars->o_full[x]));
                            }
                            __syncwarp();
                        }
                        if (!ok) break;
                        ++p_uses[x];
                        if (j + 1 < w.n[x]) {
                            scores(x, ring_smem + (size_t)k.slot * OP);
                            if (j + 2 == w.n[x] && elect_one()) mma_commit(smem_u32(&bars->q_empty[x]));
                            __syncwarp();
                        }
                    }
                    if (!ok) break;
                    if (elect_one()) {
                        mma_commit(smem_u32(&bars->empty[v.slot]));
                        if (j + 1 < n) mma_commit(smem_u32(&bars->empty[k.slot]));
                    }
                    __syncwarp();
                }
            }
            if (elect_one()) mma_commit(smem_u32(&bars->drain));
            __syncwarp();
            mbar_wait_quiet(smem_u32(&bars->drain), 0u);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        const int group = (warp >> 2) - 1, x = group >> 1, half = group & 1, q = warp & 3, r = q * 32 + lane;
        const uint32_t lanes = (uint32_t)(q * 32) << 16, s_addr = tmem + lanes + x * 128 + half * 64, o_addr = tmem + lanes + 256 + x * 128 + half * (DB * 32);
        const int my_tok = r >> p.pack_shift, my_head = r & (p.pack - 1);
        const uint64_t scale2 = pair_of(p.scale_log2, p.scale_log2);
        uint32_t s_uses = 0, o_uses = 0, met_uses = 0;
        bool ok = true;
        // The two warps of 32 rows exchange a number for each row (through an mbarrier, whose waits end). A place is written again two exchanges later: by
        // then the other warp has arrived for the one between, behind its reading of this one.
        auto other = [&](float mine, float& its) -> bool {
            const uint32_t turn = met_uses & 1u;
            bars->swap[turn][x][half][r] = mine;
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars->met[x][q]));
            const bool met = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->met[x][q]), turn, abort_flag, p.timeout_word, TO_EPILOGUE));
            ++met_uses;
            its = bars->swap[turn][x][half ^ 1][r];
            return met;
        };
        for (Walk walk(p.table, p.items, p.packs); walk.more && ok; walk.next()) {
            const Work w = work_of(walk);
            const int n = x ? w.n[1] : w.n[0];
            if (n == 0) continue;
            const int first = w.t.at + x * tok, at = first + my_tok;      // this row's token within its sequence
            float ref = -INFINITY, sum = 0.0f;               // reference of the exponents (times scale, in powers of two)
            for (int j = 0; j < n; ++j) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->s_full[x]), s_uses++ & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
                if (!ok) break;
                tc_fence_after();
                uint32_t s[2][32];
                float top2[2];
                const int key0 = (w.j0 + j) * TILE;
                const bool masked = key0 + TILE - 1 > first;      // keys behind the tile's first token: some row does not see all of them
                const int lim = at - key0 - half * 64;   // this row's last key among the 64
                tmem_ld_x32(s_addr, s[0]);
                tmem_wait_ld();
                tmem_ld_x32(s_addr + 32, s[1]);              // on its way while the first half's maximum is taken
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if (c == 1) tmem_wait_ld();
                    if (masked) {
#pragma unroll
                        for (int k = 0; k < 32; ++k) if (c * 32 + k > lim) s[c][k] = 0xFF800000u;
                    }
                    float t[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        t[h] = max3(__uint_as_float(s[c][h * 16]), __uint_as_float(s[c][h * 16 + 1]), __uint_as_float(s[c][h * 16 + 2]));
#pragma unroll
                        for (int k = 3; k + 1 < 16; k += 2) t[h] = max3(t[h], __uint_as_float(s[c][h * 16 + k]), __uint_as_float(s[c][h * 16 + k + 1]));
                    }
                    top2[c] = max3(max3(t[0], t[1], __uint_as_float(s[c][15])), __uint_as_float(s[c][31]), __uint_as_float(s[c][31]));
                }
                const float mine = max3(top2[0], top2[1], top2[1]);
                float its;
                ok = other(mine, its);
                if (!ok) break;
                const float top = max3(mine, its, its) * p.scale_log2;
                float by = 1.0f;
                if (!(top <= ref + SLACK)) {                 // (also where top is NaN: the whole row is from here on)
                    if (top != -INFINITY) {
                        by = ref == -INFINITY ? 0.0f : ex2(ref - top);
                        ref = top;
                    }
                }
                if (j > 0 && __any_sync(0xFFFFFFFFu, by != 1.0f)) {      // the products so far are complete: S was issued behind them
#pragma unroll 1
                    for (int c = 0; c < DB * 32; c += 16) {
                        uint32_t o[16];
                        tmem_ld_x16(o_addr + c, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(by == 0.0f ? 0.0f : __uint_as_float(o[k]) * by);
                        tmem_st_x16(o_addr + c, o);
                    }
                    sum *= by;
                    tmem_wait_st();
                    tc_fence_before();
                }
                if (half == 1) {                             // the first products of P may begin when both halves of O are as they have to be
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&bars->p_ready[x][0]));
                    __syncwarp();                            // (what follows in tensor memory is a whole warp's)
                }
                const float off = ref == -INFINITY ? 0.0f : ref;
                const uint64_t off2 = pair_of(-off, -off);
                uint64_t part[2] = {0, 0};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t e[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int i = c * 8 + k;
                        const uint64_t x2 = fma2(pair_of(__uint_as_float(s[i >> 4][(2 * i) & 31]), __uint_as_float(s[i >> 4][(2 * i + 1) & 31])), scale2, off2);
                        const uint64_t y2 = ex2_pair(x2);
                        part[k & 1] = add2(part[k & 1], y2);
                        e[k] = pack_pair(y2);
                    }
                    tmem_st_x8(s_addr + c * 8, e);           // over this half's own scores
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars->p_ready[x][half]));
                float pa, pb;
                split_pair(add2(part[0], part[1]), pa, pb);
                sum += pa + pb;
            }
            if (!ok) break;
            float its;
            ok = other(sum, its);
            if (!ok) break;
            sum = half ? its + sum : sum + its;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->o_full[x]), o_uses++ & 1u, abort_flag, p.timeout_word, TO_EPILOGUE));
            if (!ok) break;
            tc_fence_after();
            if (w.split) {                                   // join_kernel does what follows
                const int64_t row = (int64_t)walk.item * TILE + r;
                if (half == 0) p.stat[row] = make_float2(ref, sum);
                float4* dst = reinterpret_cast<float4*>(p.part + row * (DB * 64) + half * (DB * 32));
#pragma unroll
                for (int c = 0; c < DB * 32; c += 32) {
                    if (half * (DB * 32) + c >= p.head_dim) break;
                    uint32_t o[32];
                    __syncwarp();
                    tmem_ld_x32(o_addr + c, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        dst[c / 4 + k] = make_float4(__uint_as_float(o[4 * k]), __uint_as_float(o[4 * k + 1]), __uint_as_float(o[4 * k + 2]), __uint_as_float(o[4 * k + 3]));
                }
                tc_fence_before();
                continue;
            }
            const float inv = 1.0f / sum;
            if (half == 0 && p.lse != nullptr && at < w.t.len) p.lse[(int64_t)(w.t.t0 + at) * p.heads + w.head0 + my_head] = (ref + log2f(sum)) * LN2;
            __nv_bfloat16* dst[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int rr = q * 32 + (lane & ~3) + k, a = first + (rr >> p.pack_shift);
                dst[k] = a < w.t.len ? p.out + (int64_t)(w.t.t0 + a) * p.ld_out + (int64_t)(w.head0 + (rr & (p.pack - 1))) * p.head_dim : nullptr;
            }
#pragma unroll
            for (int c = 0; c < DB * 32; c += 32) {
                if (half * (DB * 32) + c >= p.head_dim) break;
                uint32_t o[32];
                float f[32];
                __syncwarp();
                tmem_ld_x32(o_addr + c, o);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 32; ++k) f[k] = __uint_as_float(o[k]) * inv;
                store_rows32(f, half * (DB * 32) + c, p.head_dim, lane, dst);
            }
            tc_fence_before();                               // (read before the next tile's products, which wait for its P)
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, 512); }
}

// The pieces of a tile's keys, joined in their order: o = sum_s e^(ref_s - m) O_s / sum_s e^(ref_s - m) sum_s with the largest reference m. A warp has a row,
// a lane four columns of it; block (piece, pack, eighth of the rows), that of a tile's first piece does the tile.
template <int DB>
__global__ void __launch_bounds__(128) join_kernel(const __grid_constant__ ForwardParams p)
{
    ahead_wait();
    ahead_release();
    const AttnTile t = p.table.few[blockIdx.x];
    const int tok = TILE >> p.pack_shift, loops = (min(t.at + tok, t.len) + TILE - 1) / TILE, pieces = (loops + p.chunk - 1) / p.chunk;
    if ((t.way >> 1) != 0 || pieces == 1) return;
    const int warp = threadIdx.x >> 5, c = (threadIdx.x & 31) * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = blockIdx.z * 16 + warp * 4 + i, at = t.at + (r >> p.pack_shift), head = (int)blockIdx.y * p.pack + (r & (p.pack - 1));
        if (at >= t.len) break;
        float top = -INFINITY, sum = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < pieces; ++s) top = fmaxf(top, p.stat[((int64_t)(blockIdx.x + s) * p.packs + blockIdx.y) * TILE + r].x);
        for (int s = 0; s < pieces; ++s) {
            const int64_t row = ((int64_t)(blockIdx.x + s) * p.packs + blockIdx.y) * TILE + r;
            const float2 st = p.stat[row];
            const float by = ex2(st.x - top);                // (a piece whose keys the row does not see: 0)
            sum += by * st.y;
            if (c < p.head_dim) {
                const float4 x = *reinterpret_cast<const float4*>(p.part + row * (DB * 64) + c);
                o[0] += by * x.x; o[1] += by * x.y; o[2] += by * x.z; o[3] += by * x.w;
            }
        }
        const float inv = 1.0f / sum;
        if (p.lse != nullptr && c == 0) p.lse[(int64_t)(t.t0 + at) * p.heads + head] = (top + log2f(sum)) * LN2;
        if (c < p.head_dim)
            *reinterpret_cast<uint2*>(p.out + (int64_t)(t.t0 + at) * p.ld_out + (int64_t)head * p.head_dim + c) = make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
    }
}

struct Chunk { AttnTile t[240]; };
__global__ void table_kernel(const __grid_constant__ Chunk src, AttnTile* __restrict__ dst, int n)
{
    ahead_wait();
    ahead_release();
    if ((int)threadIdx.x < n) dst[threadIdx.x] = src.t[threadIdx.x];
}

// Tiles sorted by the length of their loops, longest first (a counting sort: loops are short numbers).
std::vector<AttnTile> longest_first(const std::vector<AttnTile>& tiles, const std::vector<int32_t>& loops, int32_t most)
{
    std::vector<int32_t> place((size_t)most + 2, 0);
    for (int32_t n : loops) ++place[(size_t)(most - n) + 1];
    for (size_t i = 1; i < place.size(); ++i) place[i] += place[i - 1];
    std::vector<AttnTile> out(tiles.size());
    for (size_t i = 0; i < tiles.size(); ++i) out[(size_t)place[(size_t)(most - loops[i])]++] = tiles[i];
    return out;
}

}  // namespace

std::vector<AttnTile> query_tiles(const AttnArgs& a, int32_t tokens_per_tile)
{
    std::vector<AttnTile> tiles;
    std::vector<int32_t> loops;
    int32_t most = 1;
    for (int64_t e = 0; e < a.n; ++e) {
        const int64_t len = a.offsets[e + 1] - a.offsets[e];
        for (int64_t at = 0; at < len; at += tokens_per_tile) {
            tiles.push_back({(int32_t)a.offsets[e], (int32_t)len, (int32_t)at, 0});
            const int32_t n = (int32_t)((std::min(at + tokens_per_tile, len) + TILE - 1) / TILE);
            loops.push_back(n);
            most = std::max(most, n);
        }
    }
    return longest_first(tiles, loops, most);
}

std::vector<AttnTile> key_tiles(const AttnArgs& a)
{
    std::vector<AttnTile> tiles;
    std::vector<int32_t> loops;
    int32_t most = 1;
    for (int64_t e = 0; e < a.n; ++e) {
        const int64_t len = a.offsets[e + 1] - a.offsets[e];
        for (int64_t at = 0; at < len; at += TILE) {
            tiles.push_back({(int32_t)a.offsets[e], (int32_t)len, (int32_t)at, 0});
            const int32_t n = (int32_t)((len - at + TILE - 1) / TILE);
            loops.push_back(n);
            most = std::max(most, n);
        }
    }
    return longest_first(tiles, loops, most);
}

// Room for a table of tiles: none where all travel in the launch. (A sequence has at most one tile that is not full; sequences without tokens have none.)
size_t tiles_bytes(int64_t tokens, int64_t n, int64_t rows)
{
    const int64_t most = tokens / rows + std::min(tokens, n);
    return most <= INLINE ? 0 : align_up((size_t)most * sizeof(AttnTile), 256);
}

qless_status put_table(const std::vector<AttnTile>& tiles, TileTable* table, AttnTile* dev, cudaStream_t st)
{
    table->tiles = (int32_t)tiles.size();
    table->list = nullptr;
    if (tiles.size() <= (size_t)INLINE) {
        memcpy(table->few, tiles.data(), tiles.size() * sizeof(AttnTile));
        return QLESS_OK;
    }
    for (size_t i = 0; i < tiles.size(); i += 240) {         // as launch arguments: nothing of the host's is read once the call has returned
        Chunk c;
        const size_t n = std::min<size_t>(240, tiles.size() - i);
        memcpy(c.t, tiles.data() + i, n * sizeof(AttnTile));
        QLESS_CUDA_TRY(launch_ahead(table_kernel, dim3(1), dim3(256), 0, st, c, dev + i, (int)n));
        count_launches(1);
    }
    table->list = dev;
    return QLESS_OK;
}

qless_status head_map(CUtensorMap* out, const void* base, int64_t ld, int32_t heads, int32_t head_dim, int64_t tokens, uint32_t box_heads, uint32_t box_tokens)
{
    return make_tmap_heads_sw128(out, base, (uint64_t)head_dim, (uint64_t)heads, (uint64_t)tokens, (uint64_t)ld * 2, box_heads, box_tokens);
}

}  // namespace attn

using namespace attn;

static int32_t pack_shift(int32_t pack) { return pack <= 1 ? 0 : 1 + pack_shift(pack / 2); }

int32_t attn_pack(int32_t heads, int32_t kv_heads)
{
    const int32_t group = heads / kv_heads;
    int32_t pack = 1;
    while (pack < 16 && group % (2 * pack) == 0) pack *= 2;
    return pack;
}

// Room for the pieces' sums, wherever some examples of so many tokens may want it: whether tiles are dealt out, and in how large pieces, follows from the whole list
// of the call's lengths, the head counts and the number of SMs, and so does the order of the sums: the same list gives the same bits wherever the examples lie and whatever
// the others hold; beside other lengths an example's sums may be cut elsewhere. (The backward pass leaves two sums of a row, and its longest loop is that over the query rows of a tile of keys.)
size_t attn::split_bytes(int64_t tokens, int32_t heads, int32_t kv_heads, bool backward)
{
    const int32_t pack = attn_pack(heads, kv_heads);
    const int64_t steps = backward ? (tokens / (TILE / pack) + 1) * (heads / kv_heads / pack) : tokens / TILE + 1;
    if (steps <= (backward ? SPLIT_BACKWARD : SPLIT_FORWARD)) return 0;
    return (size_t)SPLIT_ROUNDS * sm_count() * TILE * (sizeof(float2) + (backward ? 256 : 128) * sizeof(float));
}

// Deals the tiles out in pieces of so many steps of their loops as it returns; 0: not worth it. per: items of a tile; gain: what has to come off.
int32_t attn::split_tiles(std::vector<AttnTile>* tiles, int32_t per, int32_t gain, const std::function<int32_t(const AttnTile&)>& loops)
{
    if (tiles->size() > (size_t)INLINE || (int64_t)tiles->size() * per > SPLIT_ROUNDS * sm_count()) return 0;
    std::vector<int32_t> n;
    int32_t most = 0, best = 0;
    for (const AttnTile& t : *tiles) { n.push_back(loops(t)); most = std::max(most, n.back()); }
    auto fits = [&](int32_t chunk, int32_t rounds) {
        int64_t pieces = 0;
        for (int32_t x : n) pieces += (x + chunk - 1) / chunk;
        return pieces <= INLINE && pieces * per <= (int64_t)rounds * sm_count();
    };
    int32_t least = most + 2 - std::max(gain, most / 20 * 3);      // (a piece costs about two steps beside its own)
    for (int32_t rounds = 1; rounds <= SPLIT_ROUNDS; ++rounds) {
        int32_t lo = 1, hi = least / rounds - 2;             // the smallest that fits
        if (hi < lo || !fits(hi, rounds)) continue;
        while (lo < hi) {
            const int32_t mid = lo + (hi - lo) / 2;
            if (fits(mid, rounds)) hi = mid;
            else lo = mid + 1;
        }
        least = rounds * (lo + 2) - 1;
        best = lo;
    }
    if (best == 0) return 0;
    std::vector<AttnTile> out;
    for (size_t i = 0; i < n.size(); ++i)
        for (int32_t j = 0; j < n[i]; j += best) { out.push_back((*tiles)[i]); out.back().way = j; }
    tiles->swap(out);
    return best;
}

template <int DB>
static qless_status launch_forward(const AttnArgs& a, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, ForwardParams& p, cudaStream_t st)
{
    const size_t op = (size_t)DB * 16384, budget = 227 * 1024 - 1024 - sizeof(Bars) - 2 * op;
    p.stages = (int32_t)std::min<size_t>(MAX_STAGES, budget / op);
    const size_t smem = 1024 + (2 + p.stages) * op + sizeof(Bars);
    const int64_t grid = std::min<int64_t>(p.items, sm_count());
    ProfileScope ps("attention", st);
    QLESS_CUDA_TRY((allow_full_smem<attention_kernel<DB>>()));
    QLESS_CUDA_TRY(launch_ahead(attention_kernel<DB>, dim3((unsigned)grid), dim3(NTHREADS), smem, st, q, k, v, p));
    count_launches(1);
    if (p.chunk > 0) {
        QLESS_CUDA_TRY(launch_ahead(join_kernel<DB>, dim3((unsigned)p.table.tiles, p.packs, 8), dim3(128), 0, st, p));
        count_launches(1);
    }
    return QLESS_OK;
}

qless_status launch_attention(const AttnArgs& a, uint8_t* ws, unsigned int* timeout_word, cudaStream_t st)
{
    const int32_t pack = attn_pack(a.heads, a.kv_heads), tok = TILE / pack, packs = a.heads / pack;
    std::vector<AttnTile> tiles = query_tiles(a, 2 * tok);
    ForwardParams p;
    p.chunk = 0; p.part = nullptr; p.stat = nullptr;
    // Too few pairs of tiles for the SMs: a tile to each block (4000 tokens, 8/8 heads of 128: 64 us, in pairs 72; 16 examples of 8000 tokens in all, 16/4 heads,
    // where there are enough: 59 us, in pairs 40).
    if ((int64_t)tiles.size() * packs < sm_count()) {
        tiles = query_tiles(a, tok);
        p.chunk = split_tiles(&tiles, packs, SPLIT_FORWARD, [&](const AttnTile& t) { return (std::min(t.at + tok, t.len) + TILE - 1) / TILE; });
        for (AttnTile& t : tiles) t.way = 1 + 2 * t.way;
        if (p.chunk > 0) {
            uint8_t* room = ws + tiles_bytes(a.tokens, a.n, tok);
            p.stat = reinterpret_cast<float2*>(room); p.part = reinterpret_cast<float*>(room + (size_t)SPLIT_ROUNDS * sm_count() * TILE * sizeof(float2));
        }
    }
    if (tiles.empty()) return QLESS_OK;
    qless_status s = put_table(tiles, &p.table, reinterpret_cast<AttnTile*>(ws), st);
    if (s != QLESS_OK) return s;
    CUtensorMap q, k, v;
    if ((s = head_map(&q, a.q, a.ld_q, a.heads, a.head_dim, a.tokens, pack, tok)) != QLESS_OK) return s;
    if ((s = head_map(&k, a.k, a.ld_k, a.kv_heads, a.head_dim, a.tokens, 1, TILE)) != QLESS_OK) return s;
    if ((s = head_map(&v, a.v, a.ld_v, a.kv_heads, a.head_dim, a.tokens, 1, TILE)) != QLESS_OK) return s;
    p.out = reinterpret_cast<__nv_bfloat16*>(a.out); p.lse = a.lse; p.ld_out = a.ld_out;
    p.packs = packs; p.pack = pack; p.pack_shift = pack_shift(pack); p.group = a.heads / a.kv_heads; p.heads = a.heads; p.head_dim = a.head_dim;
    QLESS_REQUIRE((int64_t)tiles.size() * packs < MOST_ITEMS - 65536, QLESS_ERR_UNSUPPORTED, "too many tiles: %zu of %d heads", tiles.size(), packs);
    p.items = (uint32_t)(tiles.size() * packs); p.scale_log2 = a.scale * LOG2E; p.timeout_word = timeout_word;
    return a.head_dim <= 64 ? launch_forward<1>(a, q, k, v, p, st) : launch_forward<2>(a, q, k, v, p, st);
}

}  // namespace qless
