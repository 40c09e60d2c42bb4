// Gated feed-forward block with few tokens: the weights' bytes are the floor, so the weights stream past the tokens.
//
// Every product is D^T = weights x tokens^T with 128 of the weights' output features as the rows of a tile and all tokens (up to 256) as its columns: the tensor
// core's work goes to tokens that exist, and a block reads its part of the weights once. The stages of all tiles (128 of the contraction each), one tile behind
// the other, are dealt out evenly: block c has stages c R .. (c + 1) R - 1, so every SM streams the same bytes whatever the sizes. A tile that
// several blocks share is left as that many fp32 partial sums (they stay in L2); few_finish_kernel adds a tile's in order and applies what follows the
// product. Where that costs more than it gains (short contractions, few tiles: share_of), blocks have whole tiles and what follows the product is done in
// their epilogue: two launches instead of four. No atomics.
//   GLU        forward   [g; u] = [Wg; Wu] x^T (both rows of a feature in one tile, in stages of 64), then h (g, u)
//   OUT        forward   y = Wd h^T;  backward  dx = Wg^T dg^T + Wu^T du^T;  then bf16
//   GLU_BACK   backward  dh = Wd^T dy^T, then dg, du (h)
// Bound: the weights' bytes. 61 tokens x 4096 x 11008 forward: 58 to 61 us: gate and up 37 us (whole tiles, 4.9 TB/s), down 21 us (shares, 4.3 TB/s), its join 5.4 us.
// Blocks are single CTAs: warp 0 TMA, warp 1 tcgen05, warps 2-5 epilogue; accumulators of two tiles in tensor memory (GLU beyond 128 tokens: of one).
#include <algorithm>

#include "ffn_common.cuh"

namespace qless {
namespace ffn {

namespace {

constexpr int NTHREADS = 192;
constexpr int MAX_STAGES = 6;
template <int MODE> constexpr int KB = MODE == 0 ? 64 : 128;      // contraction per stage (GLU: of both matrices)
constexpr int A_BYTES = 32768;

enum { GLU = 0, GLU_BACK = 1, OUT = 2 };

// What follows a product.
struct FinishParams {
    float* part;                            // [block's place among those that share the tile][set][tokens][feats]
    int32_t tokens, feats, act, kblocks, per;
    const __nv_bfloat16* gate_in; const __nv_bfloat16* up_in;
    __nv_bfloat16* out; __nv_bfloat16* out2; __nv_bfloat16* out3;      // GLU: h, g, u; GLU_BACK: dg, du, h; OUT: the result
    int64_t ld_gate_in, ld_up_in, ld, ld2, ld3;
};

struct FewParams {
    int32_t kswitch;                        // from this stage of a tile on: the second weights and the second tokens' operand
    int32_t n_cols, ring;                   // columns of a tile (the tokens, rounded up), places of the ring
    int32_t all, direct;                    // stages of all tiles; blocks have whole tiles and finish them
    FinishParams f;
    unsigned int* timeout_word;
};

struct __align__(8) Bars {
    uint64_t full[MAX_STAGES], empty[MAX_STAGES], d_full[2], d_empty[2], drain;
    uint32_t tmem_base, abort_flag;
};

struct Ring {
    uint32_t slot = 0, parity = 0;
    __device__ __forceinline__ void next(uint32_t n) { if (++slot == n) { slot = 0; parity ^= 1u; } }
};

// A_MN: the weights' rows in memory run along the features.
template <int MODE, bool A_MN>
__global__ void __launch_bounds__(NTHREADS, 1)
few_gemm_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_w2, const __grid_constant__ CUtensorMap tm_x,
                const __grid_constant__ CUtensorMap tm_x2, const FewParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    constexpr bool DUAL = MODE == GLU;
    constexpr int KS = KB<MODE>, BOXES = KS / 64;
    const int b_half = p.n_cols * 128, stage_bytes = A_BYTES + BOXES * b_half;      // (n_cols a multiple of 16: blocks stay on 1024-byte boundaries)
    // accumulators: of two tiles (GLU: each with the gate's at 0 and the other's at 128 columns), or the two of one
    const uint32_t bufs = DUAL && p.n_cols > 128 ? 1 : 2, second_acc = DUAL && p.n_cols > 128 ? 256 : 128;
    const uint32_t nS = (uint32_t)p.ring;
    Bars* bars = reinterpret_cast<Bars*>(smem + (size_t)nS * stage_bytes);
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < MAX_STAGES; ++s) { mbar_init(smem_u32(&bars->full[s]), 1); mbar_init(smem_u32(&bars->empty[s]), 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&bars->d_full[s]), 1); mbar_init(smem_u32(&bars->d_empty[s]), 4); }
        mbar_init(smem_u32(&bars->drain), 1);
        bars->abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tm_w); prefetch_tmap(&tm_w2); prefetch_tmap(&tm_x); prefetch_tmap(&tm_x2);
    }
    if (warp == 1) { tmem_alloc(smem_u32(&bars->tmem_base), 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;                   // accumulators at columns 0 and 256

    const int kblocks = p.f.kblocks, per = p.f.per, end = min(p.all, ((int)blockIdx.x + 1) * per);
    // The block's piece of a tile that begins at stage `at`: stages kb0 .. kb1 - 1 of the tile.
    struct Piece { int tile, place, kb0, kb1; };
    auto piece_of = [&](int at) {
        Piece x;
        x.tile = at / kblocks;
        const int begin = x.tile * kblocks;
        x.place = (int)blockIdx.x - begin / per;
        x.kb0 = at - begin;
        x.kb1 = min(kblocks, end - begin);
        return x;
    };
    // the weights of a stage: box by box (the second matrix's behind the first's, or the next 64 of the contraction)
    auto weights = [&](const Piece& x, int kb, auto each) {
        const bool second = kb >= p.kswitch;
        const int k0 = (second ? kb - p.kswitch : kb) * KS, f0 = x.tile * 128;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const CUtensorMap* m = (DUAL ? j > 0 : second) ? &tm_w2 : &tm_w;
            const int step = DUAL ? 0 : 64 * j;
            each(j, m, (A_MN ? f0 : k0) + step, A_MN ? k0 : f0);
        }
    };
    // While the kernel before this one ends: the weights of the first stages into L2 (where a write of theirs that is still to come would be seen).
    if (warp == 0) {
        int left = (int)nS;
        for (int at = blockIdx.x * per; at < end && left > 0;) {
            const Piece x = piece_of(at);
            at += x.kb1 - x.kb0;
            for (int kb = x.kb0; kb < x.kb1 && left > 0; ++kb, --left) {
                if (elect_one()) weights(x, kb, [&](int, const CUtensorMap* m, int c, int r) { tma_prefetch_2d(m, c, r); });
                __syncwarp();
            }
        }
    }
    ahead_wait();
    ahead_release();
    auto warp_wait = [&](uint64_t* bar, uint32_t parity, uint32_t code) -> bool {
        const bool w = mbar_wait(smem_u32(bar), parity, abort_flag, p.timeout_word, code);
        return __all_sync(0xFFFFFFFFu, w);
    };

    if (warp == 0) {
        Ring ring;
        uint32_t it = 0;
        bool ok = true;
        for (int at = blockIdx.x * per; at < end && ok;) {
            const Piece x = piece_of(at);
            at += x.kb1 - x.kb0;
            for (int kb = x.kb0; kb < x.kb1; ++kb, ++it, ring.next(nS)) {
                if (!warp_wait(&bars->empty[ring.slot], ring.parity ^ 1u, TO_PRODUCER)) { ok = false; break; }
                if (elect_one()) {
                    const uint32_t full = smem_u32(&bars->full[ring.slot]), a = smem_u32(smem + (size_t)ring.slot * stage_bytes), b = a + A_BYTES;
                    mbar_arrive_expect_tx(full, (uint32_t)stage_bytes);
                    weights(x, kb, [&](int j, const CUtensorMap* m, int c, int r) { tma_load_2d(a + j * 16384, m, full, c, r); });
                    const bool second = kb >= p.kswitch;
                    const int k0 = (second ? kb - p.kswitch : kb) * KS;
#pragma unroll
                    for (int j = 0; j < BOXES; ++j) tma_load_2d(b + j * b_half, second ? &tm_x2 : &tm_x, full, k0 + 64 * j, 0);
                }
                __syncwarp();
            }
        }
        if (!ok)
            for (uint32_t j = it > nS ? it - nS : 0u; j < it; ++j)
                if (!mbar_wait_quiet(smem_u32(&bars->full[j % nS]), (j / nS) & 1u, 1u << 14)) break;
    } else if (warp == 1) {
        const uint32_t idesc = make_idesc(1, 1, 1, 128, (uint32_t)p.n_cols) | (A_MN ? IDESC_A_MN : 0u);
        const uint64_t b_next = (uint64_t)(b_half / 16);      // the second 64 columns of the contraction
        Ring ring;
        uint32_t n_acc = 0;
        bool ok = true;
        for (int at = blockIdx.x * per; at < end && ok; ++n_acc) {
            const Piece x = piece_of(at);
            at += x.kb1 - x.kb0;
            const uint32_t buf = bufs == 2 ? n_acc & 1u : 0u, turn = (bufs == 2 ? n_acc >> 1 : n_acc) & 1u, d = tmem + buf * 256;
            if (!warp_wait(&bars->d_empty[buf], turn ^ 1u, TO_MMA)) { ok = false; break; }
            tc_fence_after();
            for (int kb = x.kb0; kb < x.kb1; ++kb, ring.next(nS)) {
                if (!warp_wait(&bars->full[ring.slot], ring.parity, TO_MMA)) { ok = false; break; }
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t a = smem_u32(smem + (size_t)ring.slot * stage_bytes);
                    const uint64_t a0 = A_MN ? make_smem_desc_mn_sw128(a, 16384) : make_smem_desc_sw128(a), b0 = make_smem_desc_sw128(a + A_BYTES);
                    if (DUAL) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            mma_f16_ss(d, a0 + (uint64_t)(k * 2), b0 + (uint64_t)(k * 2), idesc, kb > x.kb0 || k > 0);
                            mma_f16_ss(d + second_acc, a0 + (uint64_t)(1024 + k * 2), b0 + (uint64_t)(k * 2), idesc, kb > x.kb0 || k > 0);
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            mma_f16_ss(d, a0 + (uint64_t)(A_MN ? k * 128 : (k >> 2) * 1024 + (k & 3) * 2), b0 + (k >> 2) * b_next + (uint64_t)((k & 3) * 2), idesc,
                                       kb > x.kb0 || k > 0);
                    }
                    mma_commit(smem_u32(&bars->empty[ring.slot]));
                }
                __syncwarp();
            }
            if (ok && elect_one()) mma_commit(smem_u32(&bars->d_full[buf]));
            __syncwarp();
        }
        if (elect_one()) mma_commit(smem_u32(&bars->drain));
        __syncwarp();
        mbar_wait_quiet(smem_u32(&bars->drain), 0u);
    } else {
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        uint32_t n_acc = 0;
        for (int at = blockIdx.x * per; at < end; ++n_acc) {
            const Piece x = piece_of(at);
            at += x.kb1 - x.kb0;
            const uint32_t buf = bufs == 2 ? n_acc & 1u : 0u, turn = (bufs == 2 ? n_acc >> 1 : n_acc) & 1u, acc = tmem + lanes + buf * 256;
            const int f = x.tile * 128 + (warp & 3) * 32 + lane, tokens = p.f.tokens;
            const int64_t feats = p.f.feats;
            const bool ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars->d_full[buf]), turn, abort_flag, p.timeout_word, TO_EPILOGUE));
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int c0 = 0; c0 < tokens; c0 += 32) {
                float v[32], u[DUAL ? 32 : 1];
                load_acc(acc + c0, v);
                if constexpr (DUAL) load_acc(acc + second_acc + c0, u);
                if (f >= feats) continue;
                const int have = tokens - c0;
                if (!p.direct) {
                    float* dst = p.f.part + ((int64_t)x.place * (DUAL ? 2 : 1) * tokens + c0) * feats + f;
#pragma unroll
                    for (int k = 0; k < 32; ++k) {
                        if (k < have) dst[k * feats] = v[k];
                        if constexpr (DUAL) if (k < have) dst[(tokens + k) * feats] = u[k];
                    }
                    continue;
                }
                by_activation(p.f.act, [&](auto act) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) {
                        if (k >= have) break;
                        const int64_t t = c0 + k;
                        if constexpr (MODE == OUT) {
                            p.f.out[t * p.f.ld + f] = __float2bfloat16_rn(v[k]);
                        } else if constexpr (MODE == GLU) {
                            if (p.f.out2 != nullptr) { p.f.out2[t * p.f.ld2 + f] = __float2bfloat16_rn(v[k]); p.f.out3[t * p.f.ld3 + f] = __float2bfloat16_rn(u[k]); }
                            float a, da;
                            activation<act.value>(v[k], a, da);
                            p.f.out[t * p.f.ld + f] = __float2bfloat16_rn(a * u[k]);
                        } else {
                            const float g = __bfloat162float(p.f.gate_in[t * p.f.ld_gate_in + f]), w = __bfloat162float(p.f.up_in[t * p.f.ld_up_in + f]);
                            float a, da;
                            activation<act.value>(g, a, da);
                            p.f.out[t * p.f.ld + f] = __float2bfloat16_rn(v[k] * w * da);
                            p.f.out2[t * p.f.ld2 + f] = __float2bfloat16_rn(v[k] * a);
                            if (p.f.out3 != nullptr) p.f.out3[t * p.f.ld3 + f] = __float2bfloat16_rn(a * w);
                        }
                    }
                });
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars->d_empty[buf]));
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, 512); }
}

// Four features of a token to a thread.
template <int MODE>
__global__ void __launch_bounds__(256) few_finish_kernel(const FinishParams p)
{
    ahead_wait();
    ahead_release();
    const int quads = p.feats / 4;
    const int64_t plane = (int64_t)p.tokens * p.feats, all = (int64_t)p.tokens * quads;
    auto put = [](__nv_bfloat16* dst, const float (&v)[4]) { *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])); };
    auto get = [](const __nv_bfloat16* src, float (&v)[4]) {
        const uint2 u = *reinterpret_cast<const uint2*>(src);
        v[0] = __uint_as_float(u.x << 16); v[1] = __uint_as_float(u.x & 0xFFFF0000u); v[2] = __uint_as_float(u.y << 16); v[3] = __uint_as_float(u.y & 0xFFFF0000u);
    };
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / quads;
        const int f = (int)(i - t * quads) * 4;
        constexpr int SETS = MODE == GLU ? 2 : 1;
        float v[2][4] = {};
#pragma unroll
        for (int k = 0; k < SETS; ++k) {
            const int first = f / 128 * p.kblocks;           // the tile's first stage
            const int places = (first + p.kblocks - 1) / p.per - first / p.per + 1;
#pragma unroll 4
            for (int s = 0; s < places; ++s) {
                const float4 y = *reinterpret_cast<const float4*>(p.part + ((int64_t)s * SETS + k) * plane + t * p.feats + f);
                v[k][0] += y.x; v[k][1] += y.y; v[k][2] += y.z; v[k][3] += y.w;
            }
        }
        if (MODE == OUT) {
            put(p.out + t * p.ld + f, v[0]);
        } else if (MODE == GLU) {
            if (p.out2 != nullptr) { put(p.out2 + t * p.ld2 + f, v[0]); put(p.out3 + t * p.ld3 + f, v[1]); }
            float h[4];
            by_activation(p.act, [&](auto act) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float a, da;
                    activation<act.value>(v[0][k], a, da);
                    h[k] = a * v[1][k];
                }
            });
            put(p.out + t * p.ld + f, h);
        } else {
            float g[4], u[4], h[4];
            get(p.gate_in + t * p.ld_gate_in + f, g);
            get(p.up_in + t * p.ld_up_in + f, u);
            by_activation(p.act, [&](auto act) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float a, da;
                    activation<act.value>(g[k], a, da);
                    h[k] = a * u[k];
                    g[k] = v[0][k] * u[k] * da;
                    u[k] = v[0][k] * a;
                }
            });
            put(p.out + t * p.ld + f, g);
            put(p.out2 + t * p.ld2 + f, u);
            if (p.out3 != nullptr) put(p.out3 + t * p.ld3 + f, h);
        }
    }
}

// Stages of a block: an even share of all, at least two; or whole tiles, where their rounds are at most 30 stages longer than the even share (a stage of 32 KiB of
// weights takes a block about 0.3 us, the partial sums and the launch that joins them 8 us; 61 tokens x 4096 x 11008 forward: 60 us with whole tiles of gate and up, 63 with
// shares; 30 x 4096 x 14336: 64 and 72; 200 x 1024 x 2816, the other way: 40 and 37; 250 x 2048 x 5632 with whole tiles of the down projection too: 73, with shares 60). GLU_BACK does so for few tokens alone: its
// epilogue reads and writes five values where others write one, and a tile's 128 threads are slower at that than a kernel of its own (64 tokens x 2048 x 5632
// backward: 42 us with whole tiles, 34 with shares; 200 x 1024 x 2816: 72 and 35; 16 x 4096 x 11008: 60 and 56; 5 x 4096 x 11008: 53 and 54).
constexpr int64_t FEW_ENOUGH = 8;

struct Share { int32_t all, per, blocks, places, direct; };
template <int MODE>
Share share_of(int64_t tokens, int64_t feats, int64_t kblocks)
{
    const int64_t tiles = (feats + 127) / 128, all = tiles * kblocks, sms = sm_count();
    const int64_t rounds = (tiles + sms - 1) / sms, even = (all + sms - 1) / sms;
    if (rounds * kblocks - even <= 30 && (MODE != GLU_BACK || tokens <= FEW_ENOUGH)) {
        const int64_t per = rounds * kblocks;
        return {(int32_t)all, (int32_t)per, (int32_t)((all + per - 1) / per), 0, 1};
    }
    const int64_t per = even < 2 ? 2 : even;
    // a tile of kblocks stages lies in at most so many blocks
    return {(int32_t)all, (int32_t)per, (int32_t)((all + per - 1) / per), (int32_t)((kblocks + per - 2) / per + 1), 0};
}

int64_t blocks_of(int64_t k, int kb) { return (k + kb - 1) / kb; }

template <int MODE>
qless_status finish(const FinishParams& p, cudaStream_t st)
{
    const int64_t blocks = ((int64_t)p.tokens * (p.feats / 4) + 255) / 256;
    ProfileScope ps("ffn_finish", st);
    QLESS_CUDA_TRY(launch_ahead(few_finish_kernel<MODE>, dim3((unsigned)std::min<int64_t>(blocks, sm_count() * 8)), dim3(256), 0, st, p));
    count_launches(1);
    return QLESS_OK;
}

// k: the contraction's length; with two operands side by side (w2 behind w) twice.
template <int MODE, bool A_MN>
qless_status product(const char* name, const CUtensorMap& w, const CUtensorMap& w2, const CUtensorMap& x, const CUtensorMap& x2, int64_t k, bool twice, int32_t n_cols,
                     FinishParams f, unsigned int* timeout_word, cudaStream_t st)
{
    FewParams p{};
    p.kswitch = (int32_t)blocks_of(k, KB<MODE>);
    f.kblocks = (twice ? 2 : 1) * p.kswitch;
    const Share s = share_of<MODE>(f.tokens, f.feats, f.kblocks);
    f.per = s.per;
    p.f = f; p.n_cols = n_cols; p.all = s.all; p.direct = s.direct; p.timeout_word = timeout_word;
    const size_t stage = A_BYTES + (size_t)n_cols * 2 * KB<MODE>, budget = 227 * 1024 - 1024 - sizeof(Bars);
    p.ring = (int32_t)std::min<size_t>(MAX_STAGES, budget / stage);
    const size_t smem = 1024 + p.ring * stage + sizeof(Bars);
    { ProfileScope ps(name, st);
      QLESS_CUDA_TRY((allow_full_smem<few_gemm_kernel<MODE, A_MN>>()));
      QLESS_CUDA_TRY(launch_ahead(few_gemm_kernel<MODE, A_MN>, dim3((unsigned)s.blocks), dim3(NTHREADS), smem, st, w, w2, x, x2, p)); }
    count_launches(1);
    return s.direct ? QLESS_OK : finish<MODE>(f, st);
}

qless_status weight_map(CUtensorMap* m, const void* p, int64_t cols, int64_t rows, int64_t ld)
{
    return make_tmap_2d_sw128(m, p, 2, (uint64_t)cols, (uint64_t)rows, (uint64_t)ld * 2, 64, 128);
}
qless_status token_map(CUtensorMap* m, const void* p, int64_t cols, int64_t tokens, int64_t ld, int32_t n_cols)
{
    return make_tmap_2d_sw128(m, p, 2, (uint64_t)cols, (uint64_t)tokens, (uint64_t)ld * 2, 64, (uint32_t)n_cols);
}

}  // namespace

#define QLESS_STEP(expr)                         \
    do {                                         \
        const qless_status s__ = (expr);         \
        if (s__ != QLESS_OK) return s__;         \
    } while (0)

size_t few_workspace(int64_t tokens, int32_t width, int32_t inner, bool backward)
{
    const size_t first = backward ? (size_t)share_of<GLU_BACK>(tokens, inner, blocks_of(width, KB<GLU_BACK>)).places : (size_t)2 * share_of<GLU>(tokens, inner, blocks_of(width, KB<GLU>)).places;
    const size_t second = (size_t)share_of<OUT>(tokens, width, (backward ? 2 : 1) * blocks_of(inner, KB<OUT>)).places;
    return align_up((size_t)tokens * 4 * std::max(first * inner, second * width), 256);
}

qless_status launch_few_forward(const FfnArgs& a, uint8_t* ws, unsigned int* timeout_word, cudaStream_t st)
{
    const int32_t n_cols = (int32_t)((a.tokens + 15) / 16 * 16);
    CUtensorMap x, wg, wu, wd, h;
    QLESS_STEP(token_map(&x, a.x, a.width, a.tokens, a.ld_x, n_cols));
    QLESS_STEP(token_map(&h, a.hidden, a.inner, a.tokens, a.ld_hidden, n_cols));
    QLESS_STEP(weight_map(&wg, a.w_gate, a.width, a.inner, a.ld_wg));
    QLESS_STEP(weight_map(&wu, a.w_up, a.width, a.inner, a.ld_wu));
    QLESS_STEP(weight_map(&wd, a.w_down, a.inner, a.width, a.ld_wd));
    FinishParams f{};
    f.part = reinterpret_cast<float*>(ws); f.tokens = (int32_t)a.tokens; f.feats = a.inner; f.act = a.act;
    f.out = reinterpret_cast<__nv_bfloat16*>(a.hidden); f.out2 = reinterpret_cast<__nv_bfloat16*>(a.gate); f.out3 = reinterpret_cast<__nv_bfloat16*>(a.up);
    f.ld = a.ld_hidden; f.ld2 = a.ld_gate; f.ld3 = a.ld_up;
    QLESS_STEP((product<GLU, false>("ffn_glu", wg, wu, x, x, a.width, false, n_cols, f, timeout_word, st)));
    f.feats = a.width; f.out = reinterpret_cast<__nv_bfloat16*>(a.out); f.ld = a.ld_out;
    return product<OUT, false>("ffn_down", wd, wd, h, h, a.inner, false, n_cols, f, timeout_word, st);
}

qless_status launch_few_backward(const FfnArgs& a, __nv_bfloat16* hidden, uint8_t* ws, unsigned int* timeout_word, cudaStream_t st)
{
    const int32_t n_cols = (int32_t)((a.tokens + 15) / 16 * 16);
    CUtensorMap dy, wg, wu, wd, dg, du;
    QLESS_STEP(token_map(&dy, a.dy, a.width, a.tokens, a.ld_dy, n_cols));
    QLESS_STEP(token_map(&dg, a.gate, a.inner, a.tokens, a.ld_gate, n_cols));
    QLESS_STEP(token_map(&du, a.up, a.inner, a.tokens, a.ld_up, n_cols));
    QLESS_STEP(weight_map(&wg, a.w_gate, a.width, a.inner, a.ld_wg));
    QLESS_STEP(weight_map(&wu, a.w_up, a.width, a.inner, a.ld_wu));
    QLESS_STEP(weight_map(&wd, a.w_down, a.inner, a.width, a.ld_wd));
    FinishParams f{};
    f.part = reinterpret_cast<float*>(ws); f.tokens = (int32_t)a.tokens; f.feats = a.inner; f.act = a.act;
    f.gate_in = reinterpret_cast<const __nv_bfloat16*>(a.gate_in); f.up_in = reinterpret_cast<const __nv_bfloat16*>(a.up_in);
    f.ld_gate_in = a.ld_gate_in; f.ld_up_in = a.ld_up_in;
    f.out = reinterpret_cast<__nv_bfloat16*>(a.gate); f.out2 = reinterpret_cast<__nv_bfloat16*>(a.up); f.out3 = hidden;
    f.ld = a.ld_gate; f.ld2 = a.ld_up; f.ld3 = a.inner;
    QLESS_STEP((product<GLU_BACK, true>("ffn_glu_back", wd, wd, dy, dy, a.width, false, n_cols, f, timeout_word, st)));
    if (a.out == nullptr) return QLESS_OK;
    f.feats = a.width; f.out = reinterpret_cast<__nv_bfloat16*>(a.out); f.ld = a.ld_out;
    return product<OUT, true>("ffn_grad_x", wg, wu, dg, du, a.inner, true, n_cols, f, timeout_word, st);
}

}  // namespace ffn
}  // namespace qless
