// Softmax cross entropy of a language model's head over a large vocabulary, with its gradient; the logits are never kept.
//
//   l_tv = <h_t, W_v>;  loss_t = logsumexp_v l_tv - l_t,y;  dh_t = w_t (sum_v p_tv W_v - W_y);  dW_v = sum_t w_t (p_tv - [v = y_t]) h_t
//
// The label's column is kept apart from the others. With s = sum_{v != y} exp(l_v - r) for some reference r:
//   d = r + log s - l_y,  loss = log(1 + e^d),  1 - p_y = sigma(d),  dh = w sigma(d) (sum_{v != y} exp(l_v - r) W_v / s - W_y):
// no difference of nearly equal numbers is formed for a token the model is sure of. In dh the label's factor w sigma(d), on which the length of
// the whole row hangs, keeps its 24 bits: alone, dh has it outside the product; with dW the product's operand holds it rounded to bf16, and
// loss_finish_kernel adds what the rounding took, times W_y. In dW it is rounded to bf16 (2^-8 of itself) like the other probabilities: a row
// of dW would have to find the tokens that carry its label. Everything is kept in powers of two (l * log2 e).
//
// Tokens without a label inside [0, V) take no part: the others are gathered first (their number stays on the device), so that an
// infinity or NaN in an ignored row meets no product, and ignored tokens cost nothing.
//
// All products run in one kernel (head_gemm_kernel, tcgen05 on CTA pairs, 256 x 256 tiles, bf16 operands, fp32 accumulators in
// tensor memory, two of them so that the epilogue of a tile overlaps the next tile's products):
//   STATS   h W^T        epilogue: per row and 128 columns the maximum and the sum of exponentials          (loss alone)
//   PROBS   h W^T        epilogue: exp(l - r) or w (p - [v = y]) as bf16 into one piece of the vocabulary    (gradients)
//   GRAD_H  piece * W    epilogue: fp32, added to what the earlier pieces left
//   GRAD_W  piece^T * h  epilogue: bf16 rows of dW
// Up to FEW = 192 tokens the roles of rows and columns are swapped (256 rows of W, or hidden channels, by all tokens): with the tokens
// as the 256 rows of a tile most of the tensor pipe's work would go to rows that do not exist, and takes longer than W's bytes. The swapped epilogue
// exchanges a row's partial sums between lanes, which costs more the more tokens there are (hidden states' gradient, swapped against not:
// 64 tokens x 4096 x 32001 138 for 157 us, 128 tokens 147 for 164, 192 tokens 161 for 165, 224 tokens 168 for 166, 256 tokens 177 for 171;
// x 2048 x 50021: 96 tokens 127 for 134 us, 160 tokens 144 for 143, 192 tokens 151 for 146, 224 tokens 169 for 156).
// Gradient of the hidden states alone: two products instead of three. The reference r of a row is its label's logit, a dot product
// taken when the row is gathered. Any reference gives the same softmax, and with the exponents of fp32 and bf16 one that lies up to
// LIMIT = 64 powers of two (a loss of 44) below the row's maximum is as good as the maximum itself. Should a row exceed that, a flag
// sends all rows through a second pass whose reference is the true maximum: its launches are always enqueued and return at once
// when the flag is not set (the host does not wait to find out). A single such row, or one with an infinity, so costs the batch both products again.
// With dW the normaliser has to be known before the piece is written: STATS first, then PROBS, GRAD_H and GRAD_W per piece.
#include "qless_kernels.h"
#include "tc_common.cuh"

namespace qless {

namespace {

using namespace tc;

constexpr int NTHREADS = 320;               // warp 0 TMA, warp 1 MMA, warps 2-9 epilogue (two groups of four, 128 columns each)
constexpr int MAX_STAGES = 5;
constexpr int KB = 128;                     // K columns per stage: 64 KiB of operands per CTA
constexpr int HALF = 32768;                 // bytes of the A operand of a stage (and of B, where it has 256 columns)
constexpr int FEW = 192;                    // tokens up to which the roles are swapped
constexpr int ROOM = 256;                   // token rows that the swapped roles' sums and tables have room for
constexpr int GROUP_M = 16;                 // row tiles that share a pass over the column tiles (their operand stays in L2)
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float LIMIT = 64.0f;

enum { STATS = 0, PROBS = 1, GRAD_H = 2, GRAD_W = 3 };

struct LossMeta { int32_t count, splits, redo, unused; };

struct __align__(16) RowParam { float r2, w, wl, unused; };      // PROBS: out = w * exp2(l2 - r2), the label's column wl

struct GemmParams {
    const LossMeta* meta;
    const int32_t* gate;                    // NULL, or a flag: 0 = nothing to do
    int32_t cols;                           // columns of this launch (STATS, PROBS: vocabulary; GRAD_H, GRAD_W: hidden width)
    int32_t col0;                           // first vocabulary column of the launch (STATS, PROBS, GRAD_H: rows of W; GRAD_W: rows of dW)
    int32_t rows;                           // GRAD_W: vocabulary columns of the piece
    int32_t k;                              // contraction length (GRAD_W: the token count instead)
    int64_t tpad;
    int32_t stages, b_rows;                 // b_rows: rows of B that one CTA of the pair brings
    const int32_t* labels;                  // [tpad] of the gathered tokens
    const RowParam* rowp;
    float2* stat;                           // STATS: [entries per tile * tiles][tpad] (maximum, sum)
    float* psum;                            // PROBS: [entries per tile * tiles][tpad] sums, or NULL
    int32_t tile0;                          // tile index of the launch's first column tile in stat / psum
    __nv_bfloat16* out;                     // PROBS: piece [tpad][ld_out]; GRAD_W: rows of dW
    int64_t ld_out;
    float* acc;                             // GRAD_H: [splits][row tiles * 256][cols]
    int32_t accumulate;
    int32_t* redo;                          // PROBS: set where a row lies more than LIMIT above its reference
    int32_t a_whole, b_whole;               // operand rows are whole 128-byte blocks: one copy brings two side by side
    unsigned int* timeout_word;
};

struct __align__(8) Bars {
    uint64_t full[MAX_STAGES], empty[MAX_STAGES], d_full[2], d_empty[2], drain;
    uint32_t tmem_base, abort_flag;
    __align__(16) RowParam rowp[ROOM];      // swapped roles: of every token
    int32_t label[ROOM];
};

struct Ring {
    uint32_t slot = 0, parity = 0;
    __device__ __forceinline__ void next(uint32_t n) { if (++slot == n) { slot = 0; parity ^= 1u; } }
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const __nv_bfloat162 z = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&z);
}

// Sum (or maximum) over the 32 lanes of each of 32 values: lane L ends with that of value L, after 31 shuffles.
template <bool MAX>
__device__ __forceinline__ float across_lanes(float (&v)[32], int lane)
{
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) {
        const bool up = (lane & s) != 0;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            if (k >= s) break;
            const float give = up ? v[k] : v[k + s], keep = up ? v[k + s] : v[k];
            const float got = __shfl_xor_sync(0xFFFFFFFFu, give, s);
            v[k] = MAX ? fmaxf(keep, got) : keep + got;
        }
    }
    return v[0];
}

template <int MODE, bool SWAP>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(NTHREADS, 1)
head_gemm_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const GemmParams p)
{
    // Nothing to do: leave before there are barriers and tensor memory to give back. Gate, count and slices are the same for every thread of the grid and
    // for both CTAs of a pair, each reads them for itself: the launches before this one have ended, and the only writer among these kernels
    // sets the gate of a second pass, which has begun only because it is set.
    if (p.gate != nullptr && *p.gate == 0) return;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const int half_b = SWAP ? p.b_rows * 2 * KB : HALF;        // bytes of a stage's B operand in this CTA
    const int stage_bytes = HALF + half_b;
    Bars* bars = reinterpret_cast<Bars*>(smem + (size_t)p.stages * stage_bytes);
    const uint32_t nS = (uint32_t)p.stages;
    volatile uint32_t* abort_flag = &bars->abort_flag;
    constexpr bool A_MN = MODE == GRAD_W || (SWAP && MODE == GRAD_H), B_MN = !SWAP && (MODE == GRAD_H || MODE == GRAD_W);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int64_t pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < MAX_STAGES; ++s) { mbar_init(smem_u32(&bars->full[s]), 1); mbar_init(smem_u32(&bars->empty[s]), 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&bars->d_full[s]), 1); mbar_init(smem_u32(&bars->d_empty[s]), 16); }
        mbar_init(smem_u32(&bars->drain), 1);
        bars->abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tm_a); prefetch_tmap(&tm_b);
    }
    if (warp == 1) { tmem_alloc_pair(smem_u32(&bars->tmem_base), 512); tmem_relinquish_pair(); }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;                   // accumulators at columns 0 and 256

    const int count = p.meta->count;
    const int mt = ((MODE == GRAD_W ? p.rows : SWAP ? (count > 0 ? p.cols : 0) : count) + 255) / 256, nt = SWAP ? 1 : (p.cols + 255) / 256;
    const int splits = MODE == GRAD_H ? p.meta->splits : 1;
    const int kblocks = ((MODE == GRAD_W ? count : p.k) + KB - 1) / KB;
    const int ksplit = (kblocks + splits - 1) / splits;
    const int64_t per_split = (int64_t)mt * nt;
    const int64_t items = per_split * splits;
    // item -> (split, column tile, row tile): GROUP_M row tiles at a time, row tiles fastest
    auto item_of = [&](int64_t item, int& split, int& m, int& n, int& kb0, int& kb1) {
        split = (int)(item / per_split);
        const int64_t r = item - split * per_split;
        const int64_t g = r / ((int64_t)GROUP_M * nt);
        const int m0 = (int)g * GROUP_M, gm = min(GROUP_M, mt - m0);
        const int rest = (int)(r - g * GROUP_M * nt);
        n = rest / gm;
        m = m0 + rest - n * gm;
        kb0 = min(kblocks, split * ksplit);
        kb1 = min(kblocks, kb0 + ksplit);
    };

    // A wait of a whole warp: the same answer in every lane.
    auto warp_wait = [&](uint64_t* bar, uint32_t parity, uint32_t code) -> bool {
        const bool w = mbar_wait_cluster(smem_u32(bar), parity, abort_flag, p.timeout_word, code);
        return __all_sync(0xFFFFFFFFu, w);
    };

    if (warp == 0) {
        {
            uint32_t it = 0;
            Ring ring;
            bool ok = true;
            for (int64_t item = pair; item < items && ok; item += num_pairs) {
                int split, m, n, kb0, kb1;
                item_of(item, split, m, n, kb0, kb1);
                // (S) rows of W start at col0, (GRAD_H) its contraction does
                const int a0 = m * 256 + (int)rank * 128 + (SWAP && !A_MN ? p.col0 : 0);
                const int b0 = SWAP ? (int)rank * p.b_rows : n * 256 + (int)rank * 128 + (B_MN ? 0 : p.col0);
                for (int kb = kb0; kb < kb1; ++kb, ++it, ring.next(nS)) {
                    if (!warp_wait(&bars->empty[ring.slot], ring.parity ^ 1u, TO_PRODUCER)) { ok = false; break; }
                    const uint32_t full = map_to_cta(smem_u32(&bars->full[ring.slot]), 0);
                    const uint32_t a = smem_u32(smem + (size_t)ring.slot * stage_bytes), b = a + HALF;
                    const int k0 = kb * KB, kw = k0 + (MODE == GRAD_H ? p.col0 : 0);
                    const int ac = A_MN ? a0 : k0, ar = A_MN ? (SWAP ? kw : k0) : a0, bc = B_MN ? b0 : k0, br = B_MN ? kw : b0;      // first column and row
                    if (elect_one()) {
                        if (rank == 0) mbar_arrive_expect_tx(smem_u32(&bars->full[ring.slot]), 2 * stage_bytes);      // both CTAs' bytes
                        if (p.a_whole) tma_load_3d_pair(a, &tm_a, full, 0, ar, ac / 64);
                        else for (int j = 0; j < 2; ++j) tma_load_2d_pair(a + j * 16384, &tm_a, full, ac + 64 * j, ar);
                        if (p.b_whole) tma_load_3d_pair(b, &tm_b, full, 0, br, bc / 64);
                        else for (int j = 0; j < 2; ++j) tma_load_2d_pair(b + j * (half_b / 2), &tm_b, full, bc + 64 * j, br);
                    }
                    __syncwarp();
                }
            }
            if (ok) ok = __all_sync(0xFFFFFFFFu, ring_drained(bars->empty, ring, nS, abort_flag, p.timeout_word, TO_PRODUCER));
            if (!ok) {       // leave no copy in flight: the leader waits (bounded) for the stages that are armed, the peer idles
                if (rank == 0) {
                    for (uint32_t j = (it > nS ? it - nS : 0u); j < it; ++j)
                        if (!mbar_wait_quiet(smem_u32(&bars->full[j % nS]), (j / nS) & 1u, 1u << 14)) break;
                } else {
                    for (uint32_t t = 0; t < (1u << 14); ++t) __nanosleep(64);
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const uint32_t idesc = make_idesc(1, 1, 1, 256, SWAP ? 2 * p.b_rows : 256) | (A_MN ? IDESC_A_MN : 0u) | (B_MN ? IDESC_B_MN : 0u);
            Ring ring;
            uint32_t n_acc = 0;
            bool ok = true;
            for (int64_t item = pair; item < items && ok; item += num_pairs, ++n_acc) {
                int split, m, n, kb0, kb1;
                item_of(item, split, m, n, kb0, kb1);
                const uint32_t buf = n_acc & 1u, d = tmem + buf * 256;
                if (!warp_wait(&bars->d_empty[buf], ((n_acc >> 1) & 1u) ^ 1u, TO_MMA)) { ok = false; break; }
                tc_fence_after();
                for (int kb = kb0; kb < kb1; ++kb, ring.next(nS)) {
                    // (an own barrier that only copies arrive on: no cluster-scope acquire)
                    bool landed = mbar_wait(smem_u32(&bars->full[ring.slot]), ring.parity, abort_flag, p.timeout_word, TO_MMA);
                    landed = __all_sync(0xFFFFFFFFu, landed);
                    if (!landed) { ok = false; break; }
                    tc_fence_after();
                    if (elect_one()) {
                    const uint32_t a = smem_u32(smem + (size_t)ring.slot * stage_bytes), b = a + HALF;
                    const uint64_t b_next = (uint64_t)(half_b / 32);      // (K-major) the second 64 columns of K
                    // made once per stage, advanced by constants (units of 16 bytes)
                    const uint64_t a0 = A_MN ? make_smem_desc_mn_sw128(a, 16384) : make_smem_desc_sw128(a);
                    const uint64_t b0 = B_MN ? make_smem_desc_mn_sw128(b, 16384) : make_smem_desc_sw128(b);
                    mma_f16_ss_pair(d, a0, b0, idesc, kb > kb0);
                    const int steps = MODE == GRAD_W ? min(KB / 16, (count - kb * KB + 15) / 16) : KB / 16;      // rows behind are not cleared
#pragma unroll
                    for (int k = 1; k < KB / 16; ++k)
                        if (MODE != GRAD_W || k < steps) mma_f16_ss_pair(d, a0 + (uint64_t)(A_MN ? k * 128 : (k >> 2) * 1024 + (k & 3) * 2), b0 + (B_MN ? (uint64_t)(k * 128) : (k >> 2) * b_next + (uint64_t)((k & 3) * 2)), idesc, 1u);
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
        if (SWAP && MODE != GRAD_H) {
            for (int t = threadIdx.x - 64; t < count; t += 256) {
                bars->label[t] = p.labels[t];
                if (MODE == PROBS) bars->rowp[t] = p.rowp[t];
            }
            asm volatile("bar.sync 1, 256;" ::: "memory");
        }
        for (int64_t item = pair; SWAP && item < items; item += num_pairs, ++n_acc) {
            // lane = row of W (or hidden channel), column = token; the second group of warps takes the second half of the tokens
            int split, m, n, kb0, kb1;
            item_of(item, split, m, n, kb0, kb1);
            const int v = m * 256 + (int)rank * 128 + q * 32 + lane;
            const uint32_t buf = n_acc & 1u;
            const int lim = min(count - half * p.b_rows, p.b_rows);      // tokens of this half
            const int upto = MODE == PROBS ? min(((count + 15) & ~15) - half * p.b_rows, p.b_rows) : lim;      // (b_rows is a multiple of 16)
            bool ok = mbar_wait_cluster(smem_u32(&bars->d_full[buf]), (n_acc >> 1) & 1u, abort_flag, p.timeout_word, TO_EPILOGUE);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            tc_fence_after();
            float run_max = -INFINITY;
#pragma unroll 1
            for (int c0 = 0; c0 < upto; c0 += 32) {
                uint32_t raw[32];
                tmem_ld_x32(tmem + lane_base + buf * 256 + half * p.b_rows + c0, raw);
                tmem_wait_ld();
                const int t0 = half * p.b_rows + c0, have = lim - c0;
                if (MODE == GRAD_H) {
                    if (v < p.cols) {
                        float* dst = p.acc + ((int64_t)split * ROOM + t0) * p.cols + v;
#pragma unroll
                        for (int k = 0; k < 32; ++k) {
                            if (k >= have) break;
                            float x = kb0 == kb1 ? 0.0f : __uint_as_float(raw[k]);
                            if (p.accumulate) x += dst[(int64_t)k * p.cols];
                            dst[(int64_t)k * p.cols] = x;
                        }
                    }
                    continue;
                }
                float e[32];
                const int64_t entry = ((int64_t)(p.tile0 + m) * 2 + rank) * 4 + q;
                if (MODE == STATS) {
                    float top[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k) {
                        const bool out = k >= have || v >= p.cols || (k < have && bars->label[t0 + k] == p.col0 + v);
                        e[k] = out ? -INFINITY : __uint_as_float(raw[k]) * LOG2E;
                        top[k] = e[k];
                    }
                    const float most = across_lanes<true>(top, lane), ref = most > -INFINITY ? most : 0.0f;
#pragma unroll
                    for (int k = 0; k < 32; ++k) e[k] = ex2(e[k] - __shfl_sync(0xFFFFFFFFu, ref, k));
                    const float sum = across_lanes<false>(e, lane);
                    if (lane < have) p.stat[entry * p.tpad + t0 + lane] = make_float2(most, sum);
                } else {
                    __nv_bfloat16* dst = p.out + (int64_t)t0 * p.ld_out + v;
#pragma unroll
                    for (int k = 0; k < 32; ++k) {
                        if (k < have) {
                            const RowParam rp = bars->rowp[t0 + k];
                            const bool own = bars->label[t0 + k] == p.col0 + v, out = own || v >= p.cols;
                            const float x = out ? -INFINITY : fmaf(__uint_as_float(raw[k]), LOG2E, -rp.r2);
                            run_max = fmaxf(run_max, x);
                            e[k] = ex2(x);
                            dst[(int64_t)k * p.ld_out] = __float2bfloat16_rn(own ? rp.wl : e[k] * rp.w);
                        } else {
                            e[k] = 0.0f;
                            // GRAD_W contracts over steps of 16 tokens
                            if (c0 + k < upto) dst[(int64_t)k * p.ld_out] = __float2bfloat16_rn(0.0f);
                        }
                    }
                    if (p.psum != nullptr) {
                        const float sum = across_lanes<false>(e, lane);
                        if (lane < have) p.psum[entry * p.tpad + t0 + lane] = sum;
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_leader_tmem(smem_u32(&bars->d_empty[buf]), rank);
            if (MODE == PROBS && p.psum != nullptr && run_max > LIMIT) *p.redo = 1;
        }
        for (int64_t item = pair; !SWAP && item < items; item += num_pairs, ++n_acc) {
            int split, m, n, kb0, kb1;
            item_of(item, split, m, n, kb0, kb1);
            const int64_t row = (int64_t)m * 256 + rank * 128 + q * 32 + lane;
            const int c_lo = n * 256 + half * 128;               // first of this thread's 128 columns within the launch
            const uint32_t buf = n_acc & 1u;
            const uint32_t taddr = tmem + lane_base + buf * 256 + half * 128;
            int lab = -1;                                        // the label's place among the 128 columns
            RowParam rp = {0.0f, 0.0f, 0.0f, 0.0f};
            if (MODE == STATS || MODE == PROBS) {
                if (row < count) {
                    lab = p.labels[row] - p.col0 - c_lo;
                    if (MODE == PROBS) rp = p.rowp[row];
                }
            }
            bool ok = mbar_wait_cluster(smem_u32(&bars->d_full[buf]), (n_acc >> 1) & 1u, abort_flag, p.timeout_word, TO_EPILOGUE);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            tc_fence_after();
            float run_max = -INFINITY, run_sum = 0.0f;
#pragma unroll 1
            for (int c0 = 0; c0 < 128; c0 += 32) {
                uint32_t v[32];
                tmem_ld_x32(taddr + c0, v);
                tmem_wait_ld();
                if (c0 == 96) {                                  // this warp's share of the accumulator is read
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_leader_tmem(smem_u32(&bars->d_empty[buf]), rank);
                }
                const int have = p.cols - (c_lo + c0);           // valid columns from here on
                if (MODE == STATS || MODE == PROBS) {
                    const int lk = lab - c0;
                    const bool mine = lk >= 0 && lk < 32 && lk < have;
                    if (__any_sync(0xFFFFFFFFu, mine)) {
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (mine && k == lk) v[k] = 0xFF800000u;      // -infinity: no part of the sum over the others
                    }
                    if (have < 32) {
#pragma unroll
                        for (int k = 0; k < 32; ++k) if (k >= have) v[k] = 0xFF800000u;
                    }
                    if (MODE == STATS) {
                        float top = -INFINITY;
#pragma unroll
                        for (int k = 0; k < 32; ++k) top = fmaxf(top, __uint_as_float(v[k]));
                        top *= LOG2E;
                        const float now = fmaxf(run_max, top);
                        if (now > -INFINITY) {
                            run_sum *= ex2(run_max - now);
#pragma unroll
                            for (int k = 0; k < 32; ++k) run_sum += ex2(fmaf(__uint_as_float(v[k]), LOG2E, -now));
                            run_max = now;
                        } else {                                 // nothing but -infinity so far (or NaN, which the sum has to show)
#pragma unroll
                            for (int k = 0; k < 32; ++k) if (isnan(__uint_as_float(v[k]))) run_sum = NAN;
                        }
                    } else {
                        float e[32];
#pragma unroll
                        for (int k = 0; k < 32; ++k) {
                            const float x = fmaf(__uint_as_float(v[k]), LOG2E, -rp.r2);
                            run_max = fmaxf(run_max, x);
                            e[k] = ex2(x);
                            run_sum += e[k];
                            e[k] *= rp.w;
                        }
                        if (__any_sync(0xFFFFFFFFu, mine)) {
#pragma unroll
                            for (int k = 0; k < 32; ++k) if (mine && k == lk) e[k] = rp.wl;
                        }
                        if (row >= count) {
#pragma unroll
                            for (int k = 0; k < 32; ++k) e[k] = 0.0f;
                        }
                        uint4 w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            w[k] = make_uint4(pack_bf16(e[8 * k], e[8 * k + 1]), pack_bf16(e[8 * k + 2], e[8 * k + 3]),
                                              pack_bf16(e[8 * k + 4], e[8 * k + 5]), pack_bf16(e[8 * k + 6], e[8 * k + 7]));
                        transpose4(w, lane);
                        __nv_bfloat16* dst = p.out + (row - (lane & 3)) * p.ld_out + c_lo + c0 + (lane & 3) * 8;
#pragma unroll
                        for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(dst + k * p.ld_out) = w[k];
                    }
                } else if (MODE == GRAD_H) {
                    float* base = p.acc + ((int64_t)split * mt * 256 + row - (lane & 3)) * p.cols + c_lo + c0 + (lane & 3) * 4;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {                // 16 columns at a time
                        uint4 w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            w[k] = kb0 == kb1 ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(v[16 * h + 4 * k], v[16 * h + 4 * k + 1], v[16 * h + 4 * k + 2], v[16 * h + 4 * k + 3]);
                        transpose4(w, lane);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            // the width is a multiple of 8; rows up to the tile's 256 have room
                            if (16 * h + (lane & 3) * 4 >= have || row - (lane & 3) + k >= count) continue;
                            float4* dst = reinterpret_cast<float4*>(base + (int64_t)k * p.cols + 16 * h);
                            float4 x = make_float4(__uint_as_float(w[k].x), __uint_as_float(w[k].y), __uint_as_float(w[k].z), __uint_as_float(w[k].w));
                            if (p.accumulate) {
                                const float4 y = *dst;
                                x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
                            }
                            *dst = x;
                        }
                    }
                } else {
                    const bool none = kb0 == kb1;                // no token carries a loss
                    uint4 w[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int c = 8 * k;
                        w[k] = make_uint4(pack_bf16(__uint_as_float(v[c]), __uint_as_float(v[c + 1])), pack_bf16(__uint_as_float(v[c + 2]), __uint_as_float(v[c + 3])),
                                          pack_bf16(__uint_as_float(v[c + 4]), __uint_as_float(v[c + 5])), pack_bf16(__uint_as_float(v[c + 6]), __uint_as_float(v[c + 7])));
                        if (none) w[k] = make_uint4(0u, 0u, 0u, 0u);
                    }
                    transpose4(w, lane);
                    const int64_t first = row - (lane & 3);
                    __nv_bfloat16* dst = p.out + (p.col0 + first) * p.ld_out + c_lo + c0 + (lane & 3) * 8;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if ((lane & 3) * 8 < have && first + k < p.rows) *reinterpret_cast<uint4*>(dst + k * p.ld_out) = w[k];
                }
            }
            if (MODE == STATS && row < count) p.stat[((int64_t)(p.tile0 + n) * 2 + half) * p.tpad + row] = make_float2(run_max, run_sum);
            if (MODE == PROBS && row < count && p.psum != nullptr) {
                p.psum[((int64_t)(p.tile0 + n) * 2 + half) * p.tpad + row] = run_sum;
                if (run_max > LIMIT) *p.redo = 1;
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

// ---- tokens that carry a loss ------------------------------------------------------------------------------------------

// place[t] = position of token t among the tokens with a label in [0, V), or -1; order = the inverse. Every block scans all labels (they
// are few against the rows) and lists the tokens whose rows fall to it; then its warps copy a row each (or share the rows where there are few) and take the dot
// product with the label's row of W on the way. Rows land in `out` in order, zeros behind the last up to a multiple of 128 (GRAD_W contracts over the rows).
// Also how many slices the hidden-state product is cut into along the vocabulary: the fewest that keep 95 % of the CTA pairs busy, or
// the best of up to four (any number where the tiles do not fill one round), within the `cap_tiles` row tiles the workspace has room for.
struct GatherArgs {
    const int64_t* labels;
    const float* token_weight;
    const __nv_bfloat16* hidden;
    const __nv_bfloat16* weight;
    int64_t T, ld_hidden, ld_weight;
    int32_t V, width, pairs, col_tiles, cap_tiles, most_slices;
    int32_t* order; int32_t* place; int32_t* out_labels;
    float* out_weight; float* label_logit; float* loss;
    RowParam* rowp;
    __nv_bfloat16* out;
    LossMeta* meta;
};

constexpr int LIST = 512;

__global__ void __launch_bounds__(1024) loss_gather_kernel(const GatherArgs a)
{
    __shared__ int32_t warp_sum[2][32];
    __shared__ int2 list[LIST];                                  // token, place
    __shared__ int32_t list_label[LIST];
    __shared__ float dots[32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, vecs = a.width / 8;
    const int32_t grid = (int32_t)gridDim.x, me = (int32_t)blockIdx.x;
    auto put_logit = [&](int32_t at, float dot) {
        const float l2 = dot * LOG2E;
        a.label_logit[at] = l2;
        a.rowp[at] = RowParam{l2, 1.0f, 0.0f, 0.0f};
    };
    int32_t base = 0, listed = 0;                                // tokens kept so far, and how many of them fell to this block since the last flush
    auto flush = [&]() {                                         // whole block
        __syncthreads();
        int share = 1;                                           // warps to a row: all of them where there are few rows
        while (share * 2 * listed <= 32 && share < 32) share *= 2;
        for (int i = warp / share; i < listed; i += 32 / share) {
            const int2 e = list[i];
            const uint4* src = reinterpret_cast<const uint4*>(a.hidden + (int64_t)e.x * a.ld_hidden);
            const uint4* wrow = reinterpret_cast<const uint4*>(a.weight + (int64_t)list_label[i] * a.ld_weight);
            uint4* dst = reinterpret_cast<uint4*>(a.out + (int64_t)e.y * a.width);
            float dot = 0.0f;
#pragma unroll 4
            for (int c = lane + 32 * (warp % share); c < vecs; c += 32 * share) {
                const uint4 x = __ldg(src + c), w = __ldg(wrow + c);
                dst[c] = x;
                const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    dot = fmaf(__uint_as_float(xs[k] << 16), __uint_as_float(ws[k] << 16), dot);
                    dot = fmaf(__uint_as_float(xs[k] & 0xFFFF0000u), __uint_as_float(ws[k] & 0xFFFF0000u), dot);
                }
            }
#pragma unroll
            for (int s = 16; s > 0; s >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, s);
            if (share == 1 && lane == 0) put_logit(e.y, dot);
            if (share > 1 && lane == 0) dots[warp] = dot;
        }
        __syncthreads();
        if (share > 1 && (int)threadIdx.x < listed) {            // at most 16 rows, one pass: the warps' shares in order
            float dot = 0.0f;
            for (int w = 0; w < share; ++w) dot += dots[threadIdx.x * share + w];
            put_logit(list[threadIdx.x].y, dot);
        }
        __syncthreads();
        listed = 0;
    };
    int64_t y_next = (int64_t)threadIdx.x < a.T ? a.labels[threadIdx.x] : -1;
    for (int64_t t0 = 0; t0 < a.T; t0 += 1024) {
        const int64_t t = t0 + threadIdx.x, y = y_next;
        y_next = t + 1024 < a.T ? a.labels[t + 1024] : -1;
        const bool keep = y >= 0 && y < a.V;
        const uint32_t mask = __ballot_sync(0xFFFFFFFFu, keep);
        int32_t* sums = warp_sum[(t0 >> 10) & 1];                // two in turn: one barrier per step
        if (lane == 0) sums[warp] = __popc(mask);
        __syncthreads();
        const int32_t mine = sums[lane];
        int32_t upto = mine;                                     // sums over the warps up to and with warp `lane`
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) { const int32_t v = __shfl_up_sync(0xFFFFFFFFu, upto, s); if (lane >= s) upto += v; }
        const int32_t all = __shfl_sync(0xFFFFFFFFu, upto, 31);
        const int32_t at = base + __shfl_sync(0xFFFFFFFFu, upto - mine, warp) + __popc(mask & ((1u << lane) - 1u));
        if (me == 0 && t < a.T) {
            a.place[t] = keep ? at : -1;
            if (keep) {
                a.order[at] = (int32_t)t;
                a.out_labels[at] = (int32_t)y;
                a.out_weight[at] = a.token_weight != nullptr ? a.token_weight[t] : 1.0f;
            } else {
                a.loss[t] = 0.0f;
            }
        }
        // places base .. base + all - 1: those that are `me` modulo the grid
        const int32_t first = base + ((me - base % grid) + grid) % grid;
        if (keep && at % grid == me) {
            const int i = listed + (at - first) / grid;
            list[i] = make_int2((int32_t)t, at);
            list_label[i] = (int32_t)y;
        }
        base += all;
        listed += first < base ? (base - 1 - first) / grid + 1 : 0;
        if (listed + 1024 / grid + 1 > LIST) flush();          // room for another step
    }
    flush();
    const int64_t z0 = (int64_t)base * vecs, z1 = (int64_t)(base + 127) / 128 * 128 * vecs;
    for (int64_t i = z0 + (int64_t)blockIdx.x * 1024 + threadIdx.x; i < z1; i += (int64_t)gridDim.x * 1024)
        reinterpret_cast<uint4*>(a.out)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        const int mt = (base + 255) / 256, tiles = mt * a.col_tiles;
        int best = 1;
        if (mt > 0) {
            const int pairs = a.pairs, most = min(min(a.cap_tiles / mt, a.most_slices), tiles >= pairs ? 4 : pairs);
            float best_use = 0.0f;
            for (int s = 1; s <= most && best_use < 0.95f; ++s) {
                const int items = tiles * s, rounds = (items + pairs - 1) / pairs;
                const float use = (float)items / (float)(rounds * pairs);
                if (use > best_use) { best_use = use; best = s; }
            }
        }
        a.meta->count = base; a.meta->splits = best; a.meta->redo = 0;
    }
}

// ---- per-row work between the products -----------------------------------------------------------------------------------

enum { ROW_REFERENCE = 0, ROW_FROM_STATS = 1, ROW_FROM_SUMS = 2 };

struct RowArgs {
    const LossMeta* meta;
    const int32_t* gate;
    int32_t kind, entries;                  // entries: stretches of columns with a partial result
    int64_t tpad;
    const float2* stat;
    const float* psum;
    const float* label_logit;
    const float* weight;
    const int32_t* order;
    RowParam* rowp;
    float2* coef;                           // ROW_FROM_SUMS: w sigma(d), 1 / s
    float* loss;
};

// Eight rows per block, 128 threads per row that take every 128th stretch: the partial results of a row lie tpad apart, so it is
// the number of loads in flight that counts. Joined in a fixed order.
constexpr int ROWS = 8;
__global__ void __launch_bounds__(1024) loss_rows_kernel(const RowArgs a)
{
    if (a.gate != nullptr && *a.gate == 0) return;
    __shared__ float2 part[32][ROWS];
    const int r = threadIdx.x & (ROWS - 1), seg = threadIdx.x / ROWS, warp = threadIdx.x >> 5;
    const int count = a.meta->count;
    // (m, s) stands for s * 2^m; plain sums have m = 0
    auto join = [](float& m, float& s, float m2, float s2) {
        const float now = fmaxf(m, m2);
        if (now > -INFINITY) { s = s * ex2(m - now) + s2 * ex2(m2 - now); m = now; }
        else s += s2;                                        // 0, or NaN
    };
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < count; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t row = r0 + r;
        float m = -INFINITY, s = 0.0f;
        if (row < count) {
            if (a.kind == ROW_FROM_SUMS) {
#pragma unroll 4
                for (int i = seg; i < a.entries; i += 1024 / ROWS) s += a.psum[(int64_t)i * a.tpad + row];
            } else {
#pragma unroll 4
                for (int i = seg; i < a.entries; i += 1024 / ROWS) {
                    const float2 x = a.stat[(int64_t)i * a.tpad + row];
                    join(m, s, x.x, x.y);
                }
            }
        }
#pragma unroll
        for (int o = ROWS; o < 32; o <<= 1) {
            const float m2 = __shfl_xor_sync(0xFFFFFFFFu, m, o), s2 = __shfl_xor_sync(0xFFFFFFFFu, s, o);
            if (a.kind == ROW_FROM_SUMS) s += s2;
            else join(m, s, m2, s2);
        }
        __syncthreads();
        if ((threadIdx.x & 31) < ROWS) part[warp][r] = make_float2(m, s);
        __syncthreads();
        if (seg == 0 && row < count) {
            for (int j = 1; j < 32; ++j) {
                const float2 x = part[j][r];
                if (a.kind == ROW_FROM_SUMS) s += x.y;
                else join(m, s, x.x, x.y);
            }
            if (a.kind == ROW_REFERENCE) {
                a.rowp[row] = RowParam{m > -INFINITY ? m : 0.0f, 1.0f, 0.0f, 0.0f};
                continue;
            }
            const float ref = a.kind == ROW_FROM_SUMS ? a.rowp[row].r2 : m;
            const float w = a.weight[row], ly = a.label_logit[row];
            const float others = s == 0.0f ? -INFINITY : ref + log2f(s);      // no other column has any weight (or there is none)
            const float d = others - ly;
            // log(1 + e^d) and the probability of the others
            const float e = exp2f(-fabsf(d)), tail = log1pf(e);
            float nll = d > 0.0f ? d * LN2 + tail : tail;
            float sigma = d > 0.0f ? 1.0f / (1.0f + e) : e / (1.0f + e);
            if (others == -INFINITY) { nll = ly - ly; sigma = nll; }               // 0; NaN where the label's logit is infinite or NaN
            else if (d != d || ly == INFINITY) { nll = NAN; sigma = NAN; }         // (infinity - infinity)
            a.loss[a.order[row]] = nll;
            if (a.kind == ROW_FROM_SUMS) a.coef[row] = make_float2(w * sigma, s == 0.0f ? 0.0f : 1.0f / s);
            else a.rowp[row] = RowParam{fmaxf(others, ly) + tail * LOG2E, w, -w * sigma, 0.0f};      // the full normaliser
        }
    }
}

// Gradient rows of all tokens: joins the slices of the vocabulary; zero for tokens without a loss. `sums` = the accumulator holds
// sum exp2(l2 - r2) W_v over the other columns; otherwise the gradient with the label's factor rounded to bf16, whose rest is added here (error of dh
// against 64 bits, 3001 tokens x 2048 x 50021: 2.4e-3 of its norm without that, 1.7e-3 with it, which is its own rounding to bf16).
__global__ void loss_finish_kernel(const float* __restrict__ acc, int32_t width, const LossMeta* __restrict__ meta,
                                   const int32_t* __restrict__ place, const int32_t* __restrict__ labels, const float2* __restrict__ coef, const RowParam* __restrict__ rowp, int32_t sums,
                                   const __nv_bfloat16* __restrict__ weight, int64_t ld_weight, int64_t T, __nv_bfloat16* __restrict__ out, int64_t ld_out)
{
    const int vecs = width / 8, splits = meta->splits;
    const int64_t slice = (int64_t)(meta->count + 255) / 256 * 256;
    const int64_t total = T * vecs;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t t = i / vecs;
        const int c = (int)(i - t * vecs) * 8;
        const int r = place[t];
        uint4 o = make_uint4(0u, 0u, 0u, 0u);
        if (r >= 0) {
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = 0.0f;
            for (int s = 0; s < splits; ++s) {
                const float4* src = reinterpret_cast<const float4*>(acc + (s * slice + r) * width + c);
                const float4 a = src[0], b = src[1];
                x[0] += a.x; x[1] += a.y; x[2] += a.z; x[3] += a.w; x[4] += b.x; x[5] += b.y; x[6] += b.z; x[7] += b.w;
            }
            const uint4 y = *reinterpret_cast<const uint4*>(weight + (int64_t)labels[r] * ld_weight + c);
            const uint32_t yw[4] = {y.x, y.y, y.z, y.w};
            if (sums) {
                const float2 k = coef[r];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[2 * j] = k.x * (x[2 * j] * k.y - __uint_as_float(yw[j] << 16));
                    x[2 * j + 1] = k.x * (x[2 * j + 1] * k.y - __uint_as_float(yw[j] & 0xFFFF0000u));
                }
            } else {
                const float wl = rowp[r].wl, rest = wl - __bfloat162float(__float2bfloat16_rn(wl));
                auto add = [&](float& sum, float w) { const float v = rest * w; if (fabsf(v) < INFINITY) sum += v; };      // (what is not finite is in the sum)
#pragma unroll
                for (int j = 0; j < 4; ++j) { add(x[2 * j], __uint_as_float(yw[j] << 16)); add(x[2 * j + 1], __uint_as_float(yw[j] & 0xFFFF0000u)); }
            }
            o = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
        }
        *reinterpret_cast<uint4*>(out + t * ld_out + c) = o;
    }
}

// Launched in order: none of these kernels begins before the one ahead has ended, and none lets the one behind it in early (a kernel of
// another operator launched ahead begins when the last of these has ended). A chain of launches on CTA pairs that overlapped stopped, once in some
// thousand calls, for a reason that was not found.
template <typename... Params, typename... Args>
cudaError_t launch_in_order(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

unsigned grid_of(int64_t work, int threads)
{
    const int64_t blocks = (work + threads - 1) / threads, most = (int64_t)sm_count() * 8;
    return (unsigned)(blocks < 1 ? 1 : blocks < most ? blocks : most);
}

template <int MODE, bool SWAP>
qless_status launch_gemm(const char* name, const CUtensorMap& a, const CUtensorMap& b, GemmParams p, int64_t max_items, cudaStream_t st)
{
    const size_t stage = HALF + (SWAP ? (size_t)p.b_rows * 2 * KB : HALF), budget = 227 * 1024 - 1024 - sizeof(Bars);
    p.stages = (int32_t)(budget / stage < MAX_STAGES ? budget / stage : MAX_STAGES);
    const size_t smem = 1024 + p.stages * stage + sizeof(Bars);
    QLESS_CUDA_TRY((allow_full_smem<head_gemm_kernel<MODE, SWAP>>()));
    int64_t grid = sm_count() / 2 * 2;
    if (grid > 2 * max_items) grid = 2 * max_items;
    { ProfileScope ps(name, st);
      QLESS_CUDA_TRY(launch_in_order(head_gemm_kernel<MODE, SWAP>, dim3((unsigned)grid), dim3(NTHREADS), smem, st, a, b, p)); }
    count_launches(1);
    return QLESS_OK;
}

}  // namespace

LossPlan plan_loss(int64_t T, int32_t width, int32_t vocab, bool want_h, bool want_w)
{
    LossPlan pl;
    pl.tpad = (T + 255) / 256 * 256;
    const int64_t mt = pl.tpad / 256, pairs = sm_count() / 2, nt_h = (width + 255) / 256;
    const int64_t tiles_v = ((int64_t)vocab + 255) / 256;
    // The normaliser first (one more product, six launches): for the loss alone, and with the gradient of the weights. For the gradient of the
    // hidden states alone a reference that may have to be redone (nine launches, four of which leave at once): the product that it saves counts
    // from a few MB of W on, the three launches cost 3 to 4 us where there is next to no product (against the normaliser first: 1 token x 512 x 1000
    // 49.7 for 45.6 us, 33 x 512 x 4099 54.5 for 50.7, 28 x 1720 x 1079 53.4 for 54.8, 88 x 4040 x 2783 68 for 85, 64 x 4096 x 32001 137 for 176,
    // 1024 x 2048 x 32001 237 for 317).
    pl.exact = !want_h || want_w;
    // Piece of the vocabulary whose probabilities are held at once: at most 512 MiB of bf16.
    int64_t piece_tiles = ((int64_t)512 << 20) / (pl.tpad * 256 * 2);
    if (piece_tiles < 1) piece_tiles = 1;
    if (piece_tiles > tiles_v) piece_tiles = tiles_v;
    pl.piece = (int32_t)(piece_tiles * 256);
    pl.pieces = (int32_t)((tiles_v + piece_tiles - 1) / piece_tiles);
    pl.few = T <= FEW;
    pl.entries = (int32_t)((pl.few ? 8 : 2) * tiles_v);         // partial statistics: one per warp of 32 rows of W, or per 128 columns
    // Slices where there is one row tile: as many as fill the pairs, in at most 64 MiB of sums.
    int64_t cap = ((int64_t)64 << 20) / (256 * 4 * (int64_t)width);
    cap = cap < 1 ? 1 : cap > pairs ? pairs : cap;
    if (cap < 3 * mt) cap = 3 * mt;
    pl.cap_tiles = (int32_t)cap;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off += align_up(bytes, 256); return at; };
    pl.meta_off = take(sizeof(LossMeta));
    pl.order_off = take((size_t)pl.tpad * 4);
    pl.place_off = take((size_t)pl.tpad * 4);
    pl.label_off = take((size_t)pl.tpad * 4);
    pl.weight_off = take((size_t)pl.tpad * 4);
    pl.logit_off = take((size_t)pl.tpad * 4);
    pl.coef_off = take((size_t)pl.tpad * 8);
    pl.rowp_off = take((size_t)pl.tpad * sizeof(RowParam));
    pl.stat_off = take((size_t)pl.entries * pl.tpad * 8);
    pl.hidden_off = take((size_t)pl.tpad * width * 2);
    pl.piece_off = (want_h || want_w) ? take((size_t)pl.tpad * pl.piece * 2) : 0;
    pl.acc_off = want_h ? take((size_t)cap * 256 * width * 4) : 0;
    pl.total = off + 256;
    return pl;
}

qless_status launch_loss(const LossArgs& a, const LossPlan& pl, uint8_t* ws, unsigned int* timeout_word, cudaStream_t st)
{
    LossMeta* meta = reinterpret_cast<LossMeta*>(ws + pl.meta_off);
    int32_t* order = reinterpret_cast<int32_t*>(ws + pl.order_off);
    int32_t* place = reinterpret_cast<int32_t*>(ws + pl.place_off);
    int32_t* labels = reinterpret_cast<int32_t*>(ws + pl.label_off);
    float* weight = reinterpret_cast<float*>(ws + pl.weight_off);
    float* logit = reinterpret_cast<float*>(ws + pl.logit_off);
    float2* coef = reinterpret_cast<float2*>(ws + pl.coef_off);
    RowParam* rowp = reinterpret_cast<RowParam*>(ws + pl.rowp_off);
    float2* stat = reinterpret_cast<float2*>(ws + pl.stat_off);
    float* psum = reinterpret_cast<float*>(ws + pl.stat_off);       // the statistics are read before the sums are written, and again the other way round
    __nv_bfloat16* hidden = reinterpret_cast<__nv_bfloat16*>(ws + pl.hidden_off);
    __nv_bfloat16* piece = reinterpret_cast<__nv_bfloat16*>(ws + pl.piece_off);
    float* acc = reinterpret_cast<float*>(ws + pl.acc_off);
    const bool want_h = a.grad_hidden != nullptr, want_w = a.grad_weight != nullptr;
    const int64_t mt = pl.tpad / 256, nt_h = (a.width + 255) / 256;
    const int32_t tiles_v = (a.vocab + 255) / 256;

    { ProfileScope ps("loss_gather", st);
      // a block lists at most LIST of the 1024 tokens of a step: at least four blocks
      int64_t blocks = a.T < sm_count() ? a.T : sm_count();
      if (blocks < 4) blocks = 4;
      GatherArgs g{};
      g.labels = a.labels; g.token_weight = a.token_weight; g.hidden = reinterpret_cast<const __nv_bfloat16*>(a.hidden);
      g.weight = reinterpret_cast<const __nv_bfloat16*>(a.weight); g.T = a.T; g.ld_hidden = a.ld_hidden; g.ld_weight = a.ld_weight; g.V = a.vocab;
      g.width = a.width; g.pairs = sm_count() / 2; g.col_tiles = (int32_t)nt_h; g.cap_tiles = pl.cap_tiles;
      // a slice has at least three blocks of K
      const int32_t kb = ((a.vocab < pl.piece ? a.vocab : pl.piece) + KB - 1) / KB;
      g.most_slices = kb / 3 > 1 ? kb / 3 : 1; g.order = order; g.place = place;
      g.out_labels = labels; g.out_weight = weight; g.label_logit = logit; g.loss = a.loss; g.rowp = rowp; g.out = hidden; g.meta = meta;
      QLESS_CUDA_TRY(launch_in_order(loss_gather_kernel, dim3((unsigned)blocks), dim3(1024), 0, st, g)); }
    count_launches(1);

    CUtensorMap tm_x, tm_w, tm_p;
    const bool few = pl.few;
    const int32_t b_rows = few ? (int32_t)((a.T + 31) / 32 * 16) : 128;      // rows of hidden states or of the piece that one CTA brings
    qless_status s;
    const bool whole = a.width % 64 == 0;
    if ((s = whole ? make_tmap_blocks_sw128(&tm_x, hidden, 2, a.width / 64, pl.tpad, (uint64_t)a.width * 2, 128, b_rows, 2)
                   : make_tmap_2d_sw128(&tm_x, hidden, 2, a.width, pl.tpad, (uint64_t)a.width * 2, 64, b_rows)) != QLESS_OK) return s;
    if ((s = whole ? make_tmap_blocks_sw128(&tm_w, a.weight, 2, a.width / 64, a.vocab, (uint64_t)a.ld_weight * 2, 128, 128, 2)
                   : make_tmap_2d_sw128(&tm_w, a.weight, 2, a.width, a.vocab, (uint64_t)a.ld_weight * 2, 64, 128)) != QLESS_OK) return s;
    CUtensorMap tm_xg, tm_pg;                                    // GRAD_W: boxes of 128 tokens whatever their number
    if (want_w) {
        if ((s = whole ? make_tmap_blocks_sw128(&tm_xg, hidden, 2, a.width / 64, pl.tpad, (uint64_t)a.width * 2, 128, 128, 2)
                       : make_tmap_2d_sw128(&tm_xg, hidden, 2, a.width, pl.tpad, (uint64_t)a.width * 2, 64, 128)) != QLESS_OK) return s;
        if ((s = make_tmap_blocks_sw128(&tm_pg, piece, 2, pl.piece / 64, pl.tpad, (uint64_t)pl.piece * 2, 128, 128, 2)) != QLESS_OK) return s;
    }
    if (want_h || want_w)
        if ((s = make_tmap_blocks_sw128(&tm_p, piece, 2, pl.piece / 64, pl.tpad, (uint64_t)pl.piece * 2, 128, b_rows, 2)) != QLESS_OK) return s;

    GemmParams base{};
    base.meta = meta; base.tpad = pl.tpad; base.labels = labels; base.rowp = rowp; base.b_rows = b_rows; base.timeout_word = timeout_word;
    auto stats = [&](int32_t cols, const int32_t* gate) {
        GemmParams p = base;
        p.gate = gate; p.cols = cols; p.k = a.width; p.stat = stat; p.a_whole = p.b_whole = whole;
        const int64_t tiles = (cols + 255) / 256;
        return few ? launch_gemm<STATS, true>("loss_stats", tm_w, tm_x, p, tiles, st) : launch_gemm<STATS, false>("loss_stats", tm_x, tm_w, p, mt * tiles, st);
    };
    auto rows = [&](int kind, int32_t entries, const int32_t* gate) -> qless_status {
        RowArgs r{};
        r.meta = meta; r.gate = gate; r.kind = kind; r.entries = entries; r.tpad = pl.tpad; r.stat = stat; r.psum = psum; r.label_logit = logit;
        r.weight = weight; r.order = order; r.rowp = rowp; r.coef = coef; r.loss = a.loss;
        { ProfileScope ps("loss_rows", st);
          QLESS_CUDA_TRY(launch_in_order(loss_rows_kernel, dim3(grid_of(a.T, ROWS)), dim3(1024), 0, st, r)); }
        count_launches(1);
        return QLESS_OK;
    };
    auto pieces = [&](bool keep_sums, const int32_t* gate) {
        for (int32_t k = 0; k < pl.pieces; ++k) {
            const int32_t v0 = k * pl.piece;                     // (below the vocabulary; the next one's start may pass 2^31)
            const int32_t cols = a.vocab - v0 < pl.piece ? a.vocab - v0 : pl.piece;
            GemmParams p = base;
            p.gate = gate; p.cols = cols; p.col0 = v0; p.k = a.width; p.out = piece; p.ld_out = pl.piece; p.tile0 = v0 / 256;
            p.psum = keep_sums ? psum : nullptr; p.redo = &meta->redo; p.a_whole = p.b_whole = whole;
            const int64_t tiles = (cols + 255) / 256;
            qless_status e = few ? launch_gemm<PROBS, true>("loss_probs", tm_w, tm_x, p, tiles, st) : launch_gemm<PROBS, false>("loss_probs", tm_x, tm_w, p, mt * tiles, st);
            if (e != QLESS_OK) return e;
            if (want_h) {
                GemmParams g = base;
                g.gate = gate; g.cols = a.width; g.col0 = v0; g.k = cols; g.acc = acc; g.accumulate = v0 > 0;
                g.a_whole = few ? whole : 1; g.b_whole = few ? 1 : whole;
                e = few ? launch_gemm<GRAD_H, true>("loss_grad_hidden", tm_w, tm_p, g, pl.cap_tiles * nt_h, st)
                        : launch_gemm<GRAD_H, false>("loss_grad_hidden", tm_p, tm_w, g, pl.cap_tiles * nt_h, st);
                if (e != QLESS_OK) return e;
            }
            if (want_w) {
                GemmParams g = base;
                g.gate = gate; g.cols = a.width; g.rows = cols; g.col0 = v0; g.out = reinterpret_cast<__nv_bfloat16*>(a.grad_weight); g.ld_out = a.ld_grad_weight; g.a_whole = 1; g.b_whole = whole;
                e = launch_gemm<GRAD_W, false>("loss_grad_weight", tm_pg, tm_xg, g, (int64_t)((cols + 255) / 256) * nt_h, st);
                if (e != QLESS_OK) return e;
            }
        }
        return QLESS_OK;
    };

    if (pl.exact) {
        if ((s = stats(a.vocab, nullptr)) != QLESS_OK) return s;
        if ((s = rows(ROW_FROM_STATS, pl.entries, nullptr)) != QLESS_OK) return s;
        if (want_w && (s = pieces(false, nullptr)) != QLESS_OK) return s;
    } else {
        if ((s = pieces(true, nullptr)) != QLESS_OK) return s;
        if ((s = stats(a.vocab, &meta->redo)) != QLESS_OK) return s;
        if ((s = rows(ROW_REFERENCE, pl.entries, &meta->redo)) != QLESS_OK) return s;
        if ((s = pieces(true, &meta->redo)) != QLESS_OK) return s;
        if ((s = rows(ROW_FROM_SUMS, pl.entries, nullptr)) != QLESS_OK) return s;
    }
    if (want_h) {
        { ProfileScope ps("loss_finish", st);
          QLESS_CUDA_TRY(launch_in_order(loss_finish_kernel, dim3(grid_of(a.T * (a.width / 8), 256)), dim3(256), 0, st, (const float*)acc, a.width, (const LossMeta*)meta,
                                      (const int32_t*)place, (const int32_t*)labels, (const float2*)coef, (const RowParam*)rowp, (int32_t)(want_w ? 0 : 1),
                                      reinterpret_cast<const __nv_bfloat16*>(a.weight), a.ld_weight, a.T, reinterpret_cast<__nv_bfloat16*>(a.grad_hidden),
                                      a.ld_grad_hidden)); }
        count_launches(1);
    }
    return QLESS_OK;
}

}  // namespace qless
