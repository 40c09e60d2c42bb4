// Per-example LoRA gradients from 8-bit activation checkpoints.
//
//   layer: y = W x + s B A x, A [r, in], B [out, r].  With dY the gradient at y and x^ = code * 2^(step - 127):
//     U = s dY B  [T, r],   H = s x^ A^T  [T, r]                         (1) factors: one row per token
//     dA_e = U_e^T x^_e  [r, in],   dB_e = dY_e^T H_e  [out, r]          (2) outer products: sums over the tokens of example e
//   row e of the gradient matrix = [dA_e row-major | dB_e row-major].
//
// Both steps read x^ and dY once and do 2 r multiply-adds per element read: memory-bound work on the tensor cores. Measured, 128 examples of 65 536
// tokens in all, 4096 -> 4096, rank 64, bf16 gradients, in a short burst: (1) 157 us, 5.1 TB/s of codes and dY; (2) 207 us, 4.0 TB/s and 134 MB of rows
// (both together 365 us; 428 us at the clocks that a minute of such work leaves). (2) waits for its copies most of the time (converters 60 %), the
// products' issue takes 55 % of its clocks and a block of codes 1300 of the 5600 that a stage lives.
// (1) lora_factors_kernel: M = 128 tokens, K = channels. The codes go TMA -> shared memory -> registers -> tensor memory as bf16
//     (exact: a code has 8 significant bits and the step is a power of two), from where the MMA takes its A operand; dY goes TMA ->
//     MMA as stored. fp32 sums over a slice of the channels; lora_split_kernel adds the slices.
// (2) lora_outer_kernel: M = 256 channels (two accumulators of 128 that share the factor operand), K = the tokens of one chunk of an
//     example, N = r. dY feeds the MMA as stored (channel-major A operand); the codes are expanded to bf16 in shared memory in the
//     layout such an operand has. The factors U and H are fp32 sums; a bf16 operand would cut them to 8 bits, so each is split into
//     `parts` bf16 terms (2 terms: 16 bits, for bf16 gradients; 3 terms: 24 bits, for fp32 gradients) and the products of all terms
//     are added in the same fp32 accumulator.
// Tokens behind the end of a chunk share its last 64-token block: their rows are overwritten with zeros in both operands (in the
// operand alone a NaN in the neighbour example would survive as 0 * NaN).
// Examples longer than a chunk are summed in pieces (fp32, added in piece order by lora_join_kernel). No float atomics between threads: the same
// inputs give the same bits.
#include <cstring>

#include "lora_items.h"
#include "qless_kernels.h"
#include "tc_common.cuh"

namespace qless {

namespace {

using namespace tc;

constexpr int NTHREADS = 704;               // warp 0 TMA, warp 1 MMA, warps 2-17 converters, warps 18-21 epilogue
constexpr int MAX_STAGES = 4;
constexpr int BIG = 32768;                  // operand bytes of one stage that come from the activations or dY
constexpr int CH = 128;                     // (1) channels per stage
constexpr int TOK = 64;                     // (2) tokens per stage
constexpr int TILE = 256;                   // (2) channels per item
// fp32 gradients: an accumulator in tensor memory takes at most SPAN channels or tokens (half as many tokens where three terms share it), then the
// epilogue adds it to the sum so far in global memory (always the same thread; in L2). The tensor core cuts the sum's last bits at each of its steps
// of 16 instead of rounding them, so a sum's error grows with its length, one way: 8 examples of 512 tokens, 4096 -> 4096, rank 64: 1.6e-6 of the norm
// with sums taken whole, 5.4e-7 so (fp32 products elsewhere: 4.4e-7), for 125 -> 140 us with 32 examples of 16 381 tokens (spans of 256: 2.7e-7, and
// twice the additions). bf16 gradients are rounded to 8 bits and take their sums whole.
constexpr int SPAN = 512;

struct FactorParams {
    int64_t T, ld_scales;
    const uint8_t* scales;
    float* part;                            // [2][slices][T][N64]: 0 = H, 1 = U (more than one slice or span)
    __nv_bfloat16* fac;                     // [2][boxes][T][64]: column c of term q is column q * term + c (one slice)
    float scaling;
    int32_t in, out, group, nr, n64, parts, term, boxes, slices, kb_x, kb_y, stages;      // kb_*: channel blocks per slice
    int32_t y_whole, steps_whole;
    int32_t span;                           // channel blocks that one accumulator takes
    int32_t token_tiles;
    int64_t items;
    unsigned int* timeout_word;
};

constexpr int INLINE = 64;                  // pieces that travel in the launch itself

struct OuterParams {
    const LoraChunk* chunks;                // NULL: they are in `few`
    const uint8_t* scales;
    int64_t ld_scales, ld_grads, items;
    void* grads;
    float* part;                            // [slots][rank * (in + out)]
    int32_t in, out, rank, group, nr, tiles_x, tiles, stages;
    int32_t x_whole, y_whole;               // rows of the codes / of dY are whole 128-byte blocks: one copy brings several side by side
    int32_t steps_whole;                    // step bytes of 128 channels are one aligned word
    unsigned int* timeout_word;
    LoraChunk few[INLINE];
};

// codes1, dy1, a, b: step (1), boxes of 128 tokens (channels of the weights) by 128 bytes; codes2, dy2, fac: step (2), 64 tokens.
struct LoraMaps { CUtensorMap codes1, codes2, dy1, dy2, a, b, fac; };

struct __align__(8) Bars {
    uint64_t full[MAX_STAGES], empty[MAX_STAGES], ready[MAX_STAGES], read[MAX_STAGES], d_full[2], d_empty[2], drain;
    uint32_t tmem_base, abort_flag;
};

struct Ring {
    uint32_t slot = 0, parity = 0;
    __device__ __forceinline__ void next(uint32_t n) { if (++slot == n) { slot = 0; parity ^= 1u; } }
};

// Four codes -> four bf16 values code * 2^(step - 127). A byte under 0x43 is the bf16 number 128 + (low seven bits); taking
// away 128, or 256 where the sign bit is set, leaves the code exactly, and so does the product with a power of two.
__device__ __forceinline__ uint32_t codes_to_bf16x2(uint32_t pair, uint32_t step2)
{
    const uint32_t mag = pair & 0xFF7FFF7Fu, off = pair & 0xFF80FF80u;
    const __nv_bfloat162 v = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&mag), *reinterpret_cast<const __nv_bfloat162*>(&off)),
                                     *reinterpret_cast<const __nv_bfloat162*>(&step2));
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void expand4(uint32_t w, uint32_t step2, uint32_t& lo, uint32_t& hi)
{
    lo = codes_to_bf16x2(__byte_perm(w, 0x43434343u, 0x4140), step2);
    hi = codes_to_bf16x2(__byte_perm(w, 0x43434343u, 0x4342), step2);
}
// The step in both halves. 0xFF becomes NaN and not infinity, of which a code other than 0 would make an infinite value.
__device__ __forceinline__ uint32_t step_bf16x2(uint32_t byte)
{
    const uint32_t one = (byte << 7) | (((byte + 1) >> 2) & 0x40u);
    return one | (one << 16);
}

// Up to four consecutive step bytes, the first in the low byte. Volatile: requested here, a block before they are used, and not
// where the compiler sees the use. `whole`: the groups of 128 channels start at a multiple of their number of bytes in memory.
__device__ __forceinline__ uint32_t load_step_bytes(const uint8_t* p, int n, bool whole)
{
    uint32_t v = 0u;
    if (whole && n == 4) {
        asm volatile("ld.global.nc.u32 %0, [%1];" : "=r"(v) : "l"(p));
    } else if (whole && n == 2) {
        asm volatile("ld.global.nc.u16 %0, [%1];" : "=r"(v) : "l"(p));
    } else if (n == 1) {
        asm volatile("ld.global.nc.u8 %0, [%1];" : "=r"(v) : "l"(p));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) {
                uint32_t b;
                asm volatile("ld.global.nc.u8 %0, [%1];" : "=r"(b) : "l"(p + i));
                v |= b << (8 * i);
            }
    }
    return v;
}

// The leading bf16 term of two fp32 numbers, packed; what it leaves of them stays in a and b. An infinite or NaN number is its own
// term and leaves nothing.
__device__ __forceinline__ uint32_t split_term(float& a, float& b)
{
    const __nv_bfloat162 z = __floats2bfloat162_rn(a, b);
    const float x = __low2float(z), y = __high2float(z);
    a = fabsf(x) < INFINITY ? a - x : 0.0f;
    b = fabsf(y) < INFINITY ? b - y : 0.0f;
    return *reinterpret_cast<const uint32_t*>(&z);
}

// Adds in L2, without waiting for the sum that is there. Only one thread ever adds to an address, so the order is that of its program.
__device__ __forceinline__ void add_to(float* p, uint32_t v)
{
    asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" ::"l"(p), "f"(__uint_as_float(v)) : "memory");
}
__device__ __forceinline__ void add4_to(float* p, uint32_t a, uint32_t b, uint32_t c, uint32_t d)      // p: 16-byte aligned
{
    asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p), "f"(__uint_as_float(a)), "f"(__uint_as_float(b)),
                 "f"(__uint_as_float(c)), "f"(__uint_as_float(d)) : "memory");
}

__device__ __forceinline__ void init_barriers(Bars* b)
{
    for (int s = 0; s < MAX_STAGES; ++s) { mbar_init(smem_u32(&b->full[s]), 1); mbar_init(smem_u32(&b->empty[s]), 1); mbar_init(smem_u32(&b->ready[s]), 4); mbar_init(smem_u32(&b->read[s]), 4); }
    for (int s = 0; s < 2; ++s) {
        mbar_init(smem_u32(&b->d_full[s]), 1);
        mbar_init(smem_u32(&b->d_empty[s]), 4);
    }
    mbar_init(smem_u32(&b->drain), 1);
    b->abort_flag = 0;
    fence_barrier_init();
}

// The producer leaves after a failed wait: copies 0 .. it-1 have been issued; give those that may still fly a bounded wait.
__device__ __forceinline__ void drain_copies(Bars* b, uint32_t it, uint32_t stages)
{
    for (uint32_t j = (it > stages ? it - stages : 0u); j < it; ++j)
        if (!mbar_wait_quiet(smem_u32(&b->full[j % stages]), (j / stages) & 1u)) break;
}

// ---- (1) factors -------------------------------------------------------------------------------------------------------

__global__ void __launch_bounds__(NTHREADS, 1)
lora_factors_kernel(const __grid_constant__ LoraMaps maps, const FactorParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const int op_bytes = p.n64 * 256;                       // factor operand of one stage: 128 channels x n64 (or n64 x 128)
    const int stage_bytes = BIG + op_bytes;
    Bars* bars = reinterpret_cast<Bars*>(smem + (size_t)p.stages * stage_bytes);
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t nS = (uint32_t)p.stages;

    ahead_release();
    if (threadIdx.x == 0) {
        init_barriers(bars);
        prefetch_tmap(&maps.codes1); prefetch_tmap(&maps.dy1); prefetch_tmap(&maps.a); prefetch_tmap(&maps.b);
    }
    if (warp == 1) { tmem_alloc(smem_u32(&bars->tmem_base), 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    ahead_wait();
    const uint32_t tmem = bars->tmem_base;                  // accumulators at columns 0 and 128, expanded codes of stage s at 256 + 64 s

    auto item_of = [&](int64_t item, int& slice, bool& is_x, int64_t& tile, int& kb0, int& kb1) {
        const FactorItem f = factor_item(item, p.token_tiles, gridDim.x);
        slice = f.slice; is_x = f.is_x; tile = f.tile;
        const int all = ((is_x ? p.in : p.out) + CH - 1) / CH, step = is_x ? p.kb_x : p.kb_y;
        kb0 = min(all, slice * step);
        kb1 = min(all, kb0 + step);
    };

    // A wait of a whole warp: the same answer in every lane.
    auto warp_wait = [&](uint64_t* bar, uint32_t parity, uint32_t code) -> bool {
        const bool w = mbar_wait(smem_u32(bar), parity, abort_flag, p.timeout_word, code);
        return __all_sync(0xFFFFFFFFu, w);
    };

    if (warp == 0) {
        {
            uint32_t it = 0;
            Ring ring;
            bool ok = true;
            for (int64_t item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
                int slice, kb0, kb1; bool is_x; int64_t tile;
                item_of(item, slice, is_x, tile, kb0, kb1);
                for (int kb = kb0; kb < kb1; ++kb, ++it, ring.next(nS)) {
                    if (!warp_wait(&bars->empty[ring.slot], ring.parity ^ 1u, TO_PRODUCER)) { ok = false; break; }
                    const uint32_t full = smem_u32(&bars->full[ring.slot]);
                    const uint32_t big = smem_u32(smem + (size_t)ring.slot * stage_bytes), op = big + BIG;
                    if (elect_one()) {
                        if (is_x) {
                            mbar_arrive_expect_tx(full, 128 * CH + 2 * p.nr * 128);
                            tma_load_2d(big, &maps.codes1, full, kb * CH, (int32_t)(tile * 128));
                            for (int j = 0; j < 2; ++j) tma_load_2d(op + j * p.n64 * 128, &maps.a, full, kb * CH + j * 64, 0);
                        } else {
                            mbar_arrive_expect_tx(full, 2 * 128 * 128 + p.n64 * 256);
                            if (p.y_whole) tma_load_3d(big, &maps.dy1, full, 0, (int32_t)(tile * 128), kb * 2);
                            else for (int j = 0; j < 2; ++j) tma_load_2d(big + j * 16384, &maps.dy1, full, kb * CH + j * 64, (int32_t)(tile * 128));
                            for (int j = 0; j < p.n64; j += 64) tma_load_2d(op + j * 256, &maps.b, full, j, kb * CH);
                        }
                    }
                    __syncwarp();
                }
            }
            if (!ok) drain_copies(bars, it, nS);
        }
    } else if (warp == 1) {
        {
            const uint32_t idesc_x = make_idesc(1, 1, 1, 128, p.nr), idesc_y = idesc_x | IDESC_B_MN;
            Ring ring;
            uint32_t n = 0;
            bool ok = true;
            for (int64_t item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
                int slice, from, end; bool is_x; int64_t tile;
                item_of(item, slice, is_x, tile, from, end);
                for (int kb0 = from; (kb0 < end || kb0 == from) && ok; kb0 += p.span, ++n) {
                    const int kb1 = min(end, kb0 + p.span);
                    const uint32_t buf = n & 1u, d = tmem + buf * 128;
                    if (!warp_wait(&bars->d_empty[buf], ((n >> 1) & 1u) ^ 1u, TO_MMA)) { ok = false; break; }
                    tc_fence_after();
                    for (int kb = kb0; kb < kb1; ++kb, ring.next(nS)) {
                        // the converters have seen the stage's copies land before they arrive here
                        if (!warp_wait(&bars->ready[ring.slot], ring.parity, TO_MMA)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t big = smem_u32(smem + (size_t)ring.slot * stage_bytes), op = big + BIG;
                        if (elect_one()) {
                        // Descriptors are made once per stage and advanced by constants (addresses in units of 16 bytes): made anew for every
                        // product they took 180 clocks of this thread where the product takes 48.
                        if (is_x) {
                            const uint32_t a = tmem + 256 + ring.slot * 64;
                            const uint64_t b0 = make_smem_desc_sw128(op), b1 = make_smem_desc_sw128(op + p.n64 * 128);
                            mma_f16_ts(d, a, b0, idesc_x, kb > kb0);
#pragma unroll
                            for (int k = 1; k < CH / 16; ++k) mma_f16_ts(d, a + k * 8, (k < 4 ? b0 : b1) + (uint64_t)((k & 3) * 2), idesc_x, 1u);
                        } else {
                            const uint64_t a0 = make_smem_desc_sw128(big), b0 = make_smem_desc_mn_sw128(op, 16384);
                            mma_f16_ss(d, a0, b0, idesc_y, kb > kb0);
#pragma unroll
                            for (int k = 1; k < CH / 16; ++k)
                                mma_f16_ss(d, a0 + (uint64_t)((k >> 2) * 1024 + (k & 3) * 2), b0 + (uint64_t)(k * 128), idesc_y, 1u);
                        }
                        mma_commit(smem_u32(&bars->empty[ring.slot]));
                        }
                        __syncwarp();
                    }
                    if (ok && elect_one()) mma_commit(smem_u32(&bars->d_full[buf]));
                    __syncwarp();
                }
            }
            if (elect_one()) mma_commit(smem_u32(&bars->drain));               // every MMA issued above completes before tensor memory is freed
            mbar_wait_quiet(smem_u32(&bars->drain), 0u);
        }
    } else if (warp < 18) {
        // Converters: thread = token = TMEM lane; a group of four warps to each stage (there are two to four), so that the barrier round
        // trips and latencies of one block overlap the work on the others. Every block passes through them, those of dY untouched: the
        // phase of a stage's barrier that its group waits for is always the one behind the phase it saw last.
        const int row = (warp & 3) * 32 + lane;
        const uint32_t grp = (uint32_t)(warp - 2) >> 2;
        const int groups = (p.in + p.group - 1) / p.group, per = CH / p.group;
        Ring ring;
        bool ok = grp < nS;
        for (int64_t item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
            int slice, kb0, kb1; bool is_x; int64_t tile;
            item_of(item, slice, is_x, tile, kb0, kb1);
            const int64_t t = tile * 128 + row;
            const uint8_t* sc = p.scales + t * p.ld_scales;
            auto load_steps = [&](int kb) -> uint32_t {        // the step bytes of the 4, 2 or 1 groups that the 128 channels lie in
                return (is_x && t < p.T) ? load_step_bytes(sc + kb * CH / p.group, min(per, groups - kb * CH / p.group), p.steps_whole != 0) : 0u;
            };
            uint32_t ahead = 0u;
            bool loaded = false;
            for (int kb = kb0; kb < kb1 && ok; ++kb, ring.next(nS)) {
                if (ring.slot != grp) continue;
                const uint32_t step = loaded ? ahead : load_steps(kb);
                loaded = kb + (int)nS < kb1;                   // this group's next block: its steps are requested one block early
                if (loaded) ahead = load_steps(kb + (int)nS);
                ok = warp_wait(&bars->full[ring.slot], ring.parity, TO_UNPACK);
                if (!ok) break;
                if (!is_x) {
                    if (lane == 0) mbar_arrive(smem_u32(&bars->ready[ring.slot]));
                    continue;
                }
                const uint4* src = reinterpret_cast<const uint4*>(smem + (size_t)ring.slot * stage_bytes + row * CH);
                uint4 raw[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) raw[j] = src[j ^ (row & 7)];
                tc_fence_after();
                const uint32_t dst = tmem + ((uint32_t)((warp & 3) * 32) << 16) + 256 + ring.slot * 64;
#pragma unroll
                for (int q = 0; q < 4; ++q) {                  // 32 channels: 16 tensor-memory columns of two bf16 each
                    const uint32_t s2 = step_bf16x2((step >> ((q * 32 / p.group) * 8)) & 0xFFu);
                    uint32_t v[16];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint4 w = raw[2 * q + h];
                        expand4(w.x, s2, v[8 * h + 0], v[8 * h + 1]);
                        expand4(w.y, s2, v[8 * h + 2], v[8 * h + 3]);
                        expand4(w.z, s2, v[8 * h + 4], v[8 * h + 5]);
                        expand4(w.w, s2, v[8 * h + 6], v[8 * h + 7]);
                    }
                    tmem_st_x16(dst + 16 * q, v);
                }
                tmem_wait_st();
                tc_fence_before();
                fence_proxy_async_smem();                      // the raw codes were read through the generic proxy; TMA refills them
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars->ready[ring.slot]));
            }
        }
    } else {
        const int row = (warp & 3) * 32 + lane;
        uint32_t n = 0;
        bool ok = true;
        for (int64_t item = blockIdx.x; item < p.items && ok; item += gridDim.x) {
            int slice, kb0, end; bool is_x; int64_t tile;
            item_of(item, slice, is_x, tile, kb0, end);
            for (int kb = kb0; kb < end || kb == kb0; kb += p.span, ++n) {
                const uint32_t buf = n & 1u;
                ok = mbar_wait(smem_u32(&bars->d_full[buf]), (n >> 1) & 1u, abort_flag, p.timeout_word, TO_EPILOGUE);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after();
                const int64_t t = tile * 128 + row;
                const int64_t kind = is_x ? 0 : 1;
                for (int c0 = 0; c0 < p.nr; c0 += 16) {
                    uint32_t v[16];
                    tmem_ld_x16(tmem + ((uint32_t)((warp & 3) * 32) << 16) + buf * 128 + c0, v);
                    tmem_wait_ld();
                    if (end == kb0) {                              // a slice beyond the last channel block
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] = 0u;
                    }
                    if (t >= p.T) continue;
                    float* sum = p.part + ((kind * p.slices + slice) * p.T + t) * p.n64 + c0;
                    const bool last = p.slices == 1 && kb + p.span >= end;
                    if (kb > kb0 && !last) {
#pragma unroll
                        for (int j = 0; j < 16; j += 4) add4_to(sum + j, v[j], v[j + 1], v[j + 2], v[j + 3]);
                        continue;
                    }
                    if (kb > kb0) {
#pragma unroll
                        for (int j = 0; j < 16; j += 4) {
                            const float4 y = __ldcg(reinterpret_cast<const float4*>(sum + j));
                            v[j] = __float_as_uint(y.x + __uint_as_float(v[j]));
                            v[j + 1] = __float_as_uint(y.y + __uint_as_float(v[j + 1]));
                            v[j + 2] = __float_as_uint(y.z + __uint_as_float(v[j + 2]));
                            v[j + 3] = __float_as_uint(y.w + __uint_as_float(v[j + 3]));
                        }
                    }
                    if (last) {
                        float x[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) x[j] = __uint_as_float(v[j]) * p.scaling;
                        __nv_bfloat16* dst = p.fac + (kind * p.boxes * p.T + t) * 64;
                        for (int q = 0; q < p.parts; ++q)
#pragma unroll
                            for (int j = 0; j < 16; j += 8) {
                                uint32_t w[4];
#pragma unroll
                                for (int k = 0; k < 4; ++k) w[k] = split_term(x[j + 2 * k], x[j + 2 * k + 1]);
                                const int c = q * p.term + c0 + j;
                                *reinterpret_cast<uint4*>(dst + (int64_t)(c / 64) * p.T * 64 + c % 64) = make_uint4(w[0], w[1], w[2], w[3]);
                            }
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; j += 4)
                            *reinterpret_cast<uint4*>(sum + j) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars->d_empty[buf]));
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, 512); }
}

// Several channel slices: adds them, multiplies by the adapter's scale and splits the fp32 factor into `parts` bf16 terms that add up to
// it (8 bits each): fac [2][boxes][T][64], column c of term q at column q * term + c.
__global__ void lora_split_kernel(const float* __restrict__ part, __nv_bfloat16* __restrict__ fac, int64_t T, int32_t n64, int32_t nr,
                                  int32_t slices, int32_t parts, int32_t term, int32_t boxes, float scaling)
{
    const int64_t rows = 2 * T, total = rows * (n64 / 4);
    ahead_release();
    ahead_wait();
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t row = i / (n64 / 4);
        const int c = (int)(i - row * (n64 / 4)) * 4;
        if (c >= nr) continue;
        const int64_t kind = row / T, t = row - kind * T;
        const float* src = part + (kind * slices * T + t) * n64 + c;
        float4 x = *reinterpret_cast<const float4*>(src);
        for (int s = 1; s < slices; ++s) {
            const float4 y = *reinterpret_cast<const float4*>(src + (int64_t)s * T * n64);
            x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
        }
        float v[4] = {x.x * scaling, x.y * scaling, x.z * scaling, x.w * scaling};
        __nv_bfloat16* dst = fac + (kind * boxes * T + t) * 64;
        for (int q = 0; q < parts; ++q) {
            const uint32_t lo = split_term(v[0], v[1]), hi = split_term(v[2], v[3]);
            const int at = q * term + c;
            *reinterpret_cast<uint2*>(dst + (int64_t)(at / 64) * T * 64 + at % 64) = make_uint2(lo, hi);
        }
    }
}

// ---- (2) outer products ------------------------------------------------------------------------------------------------

template <typename OutT> __device__ __forceinline__ OutT to_out(float v);
template <> __device__ __forceinline__ float to_out<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 to_out<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// A warp's 16 accumulator columns [c0, c0 + 16) of the channels ch0 + lane -> dA (column of the row-major [rank, width]) or dB (rows of
// `rank` numbers), or added to what the spans before have left there. Lanes exchange pieces so that an instruction writes whole sectors, 64
// bytes of a row of dA or dB at a time where it can (bf16: 128 stores of 64 bytes for a tile of dA took 11.6 k clocks, longer than its products).
__device__ __forceinline__ void store_columns(float* dst, bool is_x, int64_t ch0, int lane, int64_t width, int c0, int rank, const uint32_t (&v)[16], bool add)
{
    if (is_x) {
        const int64_t ch = ch0 + lane;
        if (ch >= width) return;
        if (add) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c0 + j < rank) add_to(dst + (int64_t)(c0 + j) * width + ch, v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c0 + j < rank) dst[(int64_t)(c0 + j) * width + ch] = __uint_as_float(v[j]);
        }
    } else if (add) {
        float* row = dst + (ch0 + lane) * rank + c0;           // 16-byte aligned: rank is a multiple of 8
        if (ch0 + lane >= width) return;
#pragma unroll
        for (int j = 0; j < 16; j += 4)
            if (c0 + j < rank) add4_to(row + j, v[j], v[j + 1], v[j + 2], v[j + 3]);
    } else {
        uint4 w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = make_uint4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
        transpose4(w, lane);
        const int c = c0 + (lane & 3) * 4;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t ch = ch0 + (lane & ~3) + k;
            if (ch >= width || c >= rank) continue;
            *reinterpret_cast<uint4*>(dst + ch * rank + c) = w[k];
        }
    }
}
__device__ __forceinline__ void store_columns(__nv_bfloat16* dst, bool is_x, int64_t ch0, int lane, int64_t width, int c0, int rank, const uint32_t (&v)[16], bool)
{
    uint32_t a[8];                                             // columns 2 i and 2 i + 1 of this lane's channel
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const __nv_bfloat162 z = __floats2bfloat162_rn(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
        a[i] = *reinterpret_cast<const uint32_t*>(&z);
    }
    if (is_x) {
        // 8 x 8 transposes among eight lanes: afterwards lane L holds eight channels of columns L % 8 and 8 + L % 8
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, a[i], 1);
            a[i] = (lane & 1) ? __byte_perm(got, a[i], 0x7632) : __byte_perm(a[i], got, 0x5410);
        }
        uint32_t b[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool up = (lane & 2) != 0;
            const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, up ? a[2 * i] : a[2 * i + 1], 2);
            b[i][0] = up ? got : a[2 * i];
            b[i][1] = up ? a[2 * i + 1] : got;
        }
        const int64_t ch = ch0 + (lane & ~7);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bool up = (lane & 4) != 0;
            const uint32_t g0 = __shfl_xor_sync(0xFFFFFFFFu, up ? b[2 * i][0] : b[2 * i + 1][0], 4), g1 = __shfl_xor_sync(0xFFFFFFFFu, up ? b[2 * i][1] : b[2 * i + 1][1], 4);
            const uint4 o = up ? make_uint4(g0, g1, b[2 * i + 1][0], b[2 * i + 1][1]) : make_uint4(b[2 * i][0], b[2 * i][1], g0, g1);
            const int c = c0 + 8 * i + (lane & 7);
            if (ch < width && c < rank) *reinterpret_cast<uint4*>(dst + (int64_t)c * width + ch) = o;      // the width is a multiple of 16
        }
    } else {
        const bool up = (lane & 1) != 0;                       // even lanes write columns c0 .. c0 + 7 of two rows, odd ones the next eight
        uint32_t got[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) got[k] = __shfl_xor_sync(0xFFFFFFFFu, up ? a[k] : a[4 + k], 1);
        const uint4 o0 = up ? make_uint4(got[0], got[1], got[2], got[3]) : make_uint4(a[0], a[1], a[2], a[3]);
        const uint4 o1 = up ? make_uint4(a[4], a[5], a[6], a[7]) : make_uint4(got[0], got[1], got[2], got[3]);
        const int64_t ch = ch0 + (lane & ~1);
        const int c = c0 + (up ? 8 : 0);
        if (c < rank && ch < width) {                          // (the width is even)
            *reinterpret_cast<uint4*>(dst + ch * rank + c) = o0;
            *reinterpret_cast<uint4*>(dst + (ch + 1) * rank + c) = o1;
        }
    }
}

// OutT fixes the number of terms of a factor: 2 for bf16 gradients, 3 for fp32. BOXES: 64-column blocks that hold them.
template <typename OutT, int BOXES>
__global__ void __launch_bounds__(NTHREADS, 1)
lora_outer_kernel(const __grid_constant__ LoraMaps maps, const __grid_constant__ OuterParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    constexpr int PARTS = sizeof(OutT) == 4 ? 3 : 2;
    // Where all terms together have at most 128 columns they are one operand (their sums meet in the epilogue): the channel operand is
    // read from shared memory once for all of them, whose bandwidth bounds this loop. Otherwise one product per term into the same accumulator.
    // Three terms of 64 columns: the first two side by side, the third into the second's columns (it is the smaller sum and loses less to them).
    constexpr bool WIDE = BOXES <= 3;
    constexpr int TERM_BYTES = BOXES / PARTS * 8192;         // a term's boxes, where it has boxes of its own
    constexpr int boxes = BOXES;                             // factor operand: boxes of 64 columns x 64 tokens
    constexpr int stage_bytes = BIG + boxes * 8192;
    Bars* bars = reinterpret_cast<Bars*>(smem + (size_t)p.stages * stage_bytes);
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t nS = (uint32_t)p.stages;

    ahead_release();
    if (threadIdx.x == 0) {
        init_barriers(bars);
        prefetch_tmap(&maps.codes2); prefetch_tmap(&maps.dy2); prefetch_tmap(&maps.fac);
    }
    if (warp == 1) { tmem_alloc(smem_u32(&bars->tmem_base), 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    ahead_wait();
    const uint32_t tmem = bars->tmem_base;                  // accumulator of item n, sub-tile m: column (n & 1) * 256 + m * 128

    const uint32_t items = (uint32_t)p.items, step_items = gridDim.x;
    constexpr int span = sizeof(OutT) == 4 ? (BOXES == 6 ? SPAN / 2 : SPAN) : 1 << 30;
    // The items of a block, one after another (chunk k, channel tile; no divisions on the way), with the next one's chunk already requested.
    const uint32_t tiles = (uint32_t)p.tiles, last = (items - 1) / tiles, step_k = step_items / tiles, step_tile = step_items - step_k * tiles;
    struct Walk { uint32_t item, k, tile, next_k, next_tile; LoraChunk c, ahead; bool is_x; int ch0; };
    auto chunk_at = [&](uint32_t k) { return p.chunks != nullptr ? p.chunks[min(k, last)] : p.few[min(k, last)]; };
    auto look = [&](Walk& w) {
        w.is_x = (int)w.tile < p.tiles_x;
        w.ch0 = (w.is_x ? (int)w.tile : (int)w.tile - p.tiles_x) * TILE;
        w.next_k = w.k + step_k; w.next_tile = w.tile + step_tile;
        if (w.next_tile >= tiles) { w.next_tile -= tiles; ++w.next_k; }
        w.ahead = chunk_at(w.next_k);
    };
    auto first_item = [&](Walk& w) {
        w.item = blockIdx.x; w.k = w.item / tiles; w.tile = w.item - w.k * tiles;
        w.c = chunk_at(w.k);
        look(w);
    };
    auto next_item = [&](Walk& w) {
        w.item += step_items; w.k = w.next_k; w.tile = w.next_tile; w.c = w.ahead;
        look(w);
    };

    // A wait of a whole warp: the same answer in every lane.
    auto warp_wait = [&](uint64_t* bar, uint32_t parity, uint32_t code) -> bool {
        const bool w = mbar_wait(smem_u32(bar), parity, abort_flag, p.timeout_word, code);
        return __all_sync(0xFFFFFFFFu, w);
    };

    if (warp == 0) {
        {
            uint32_t it = 0;
            Ring ring;
            bool ok = true;
            Walk w;
            for (first_item(w); w.item < items && ok; next_item(w)) {
                const LoraChunk c = w.c;
                const bool is_x = w.is_x; const int ch0 = w.ch0;
                for (int t = 0; t < c.len; t += TOK, ++it, ring.next(nS)) {
                    if (!warp_wait(&bars->empty[ring.slot], ring.parity ^ 1u, TO_PRODUCER)) { ok = false; break; }
                    const uint32_t full = smem_u32(&bars->full[ring.slot]);
                    const uint32_t big = smem_u32(smem + (size_t)ring.slot * stage_bytes), op = big + BIG;
                    const int32_t row = (int32_t)(c.t0 + t);
                    if (elect_one()) {
                        mbar_arrive_expect_tx(full, (is_x ? 2 : 4) * 8192 + boxes * 8192);
                        if (is_x) {
                            if (p.x_whole) tma_load_3d(big, &maps.codes2, full, 0, row, ch0 / 128);
                            else for (int j = 0; j < 2; ++j) tma_load_2d(big + j * 8192, &maps.codes2, full, ch0 + j * 128, row);
                        } else {
                            if (p.y_whole) tma_load_3d(big, &maps.dy2, full, 0, row, ch0 / 64);
                            else for (int j = 0; j < 4; ++j) tma_load_2d(big + j * 8192, &maps.dy2, full, ch0 + j * 64, row);
                        }
                        tma_load_3d(op, &maps.fac, full, 0, row, (is_x ? 1 : 0) * boxes);      // U for the codes, H for dY
                    }
                    __syncwarp();
                }
            }
            if (!ok) drain_copies(bars, it, nS);
        }
    } else if (warp == 1) {
        {
            const uint32_t idesc = make_idesc(1, 1, 1, 128, BOXES == 3 ? 64 + p.nr : WIDE ? PARTS * p.nr : p.nr) | IDESC_A_MN | IDESC_B_MN;
            const uint32_t idesc_third = make_idesc(1, 1, 1, 128, p.nr) | IDESC_A_MN | IDESC_B_MN;
            constexpr int TERMS = BOXES == 3 ? 2 : WIDE ? 1 : PARTS;
            Ring ring;
            uint32_t n = 0;
            bool ok = true;
            Walk w;
            for (first_item(w); w.item < items && ok; next_item(w)) {
                const LoraChunk c = w.c;
                const bool is_x = w.is_x; const int ch0 = w.ch0;
                const int subs = (is_x ? p.in : p.out) - ch0 > 128 ? 2 : 1;
                for (int t0 = 0; (t0 < c.len || t0 == 0) && ok; t0 += span, ++n) {
                    const uint32_t buf = n & 1u;
                    if (!warp_wait(&bars->d_empty[buf], ((n >> 1) & 1u) ^ 1u, TO_MMA)) { ok = false; break; }
                    tc_fence_after();
                    const int end = min(c.len, t0 + span);
                    for (int t = t0; t < end; t += TOK, ring.next(nS)) {
                        if (!warp_wait(&bars->ready[ring.slot], ring.parity, TO_MMA)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t big = smem_u32(smem + (size_t)ring.slot * stage_bytes), op = big + BIG;
                        if (elect_one()) {
                        const uint64_t a0 = make_smem_desc_mn_sw128(big, 8192), b0 = make_smem_desc_mn_sw128(op, 8192);
                        for (int m = 0; m < subs; ++m) {
                            const uint64_t am = a0 + (uint64_t)(m * 1024);
                            const uint32_t d = tmem + buf * 256 + m * 128;
                            mma_f16_ss(d, am, b0, idesc, t > t0);
#pragma unroll
                            for (int i = 1; i < TOK / 16 * TERMS; ++i) {
                                const int k = i / TERMS, q = i % TERMS;
                                if (BOXES == 3 && q == 1) mma_f16_ss(d + 64, am + (uint64_t)(k * 128), b0 + (uint64_t)(k * 128 + 2 * (TERM_BYTES / 16)), idesc_third, 1u);
                                else mma_f16_ss(d, am + (uint64_t)(k * 128), b0 + (uint64_t)(k * 128 + q * (TERM_BYTES / 16)), idesc, 1u);
                            }
                        }
                        mma_commit(smem_u32(&bars->empty[ring.slot]));
                        }
                        __syncwarp();
                    }
                    if (ok && elect_one()) mma_commit(smem_u32(&bars->d_full[buf]));
                    __syncwarp();
                }
            }
            if (elect_one()) mma_commit(smem_u32(&bars->drain));
            mbar_wait_quiet(smem_u32(&bars->drain), 0u);
        }
    } else if (warp < 18) {
        // Converters: a group of four warps to each stage (as above: every block passes through them, dY untouched but for the last,
        // partly filled block of a piece). A thread owns one token and 128 channels; the step bytes of its next block are requested
        // before it works on the present one.
        const int tid = (threadIdx.x - 64) & 127, tok = tid & 63, box = tid >> 6;
        const uint32_t grp = (uint32_t)(warp - 2) >> 2;
        const int groups = (p.in + p.group - 1) / p.group, per = 128 / p.group;
        // The group's blocks are every nS-th of all; `blk` is the block's place within the walk's item.
        Walk w;
        first_item(w);
        int blk = (int)grp, blocks = (w.c.len + TOK - 1) / TOK;
        auto settle = [&]() {
            while (blk >= blocks && w.item < items) {
                blk -= blocks;
                next_item(w);
                blocks = (w.c.len + TOK - 1) / TOK;
            }
        };
        auto load_steps = [&]() -> uint32_t {
            const int g0 = (w.ch0 + box * 128) / p.group, t = blk * TOK + tok;
            return (w.item < items && w.is_x && t < w.c.len)
                       ? load_step_bytes(p.scales + (w.c.t0 + t) * p.ld_scales + g0, min(per, groups - g0), p.steps_whole != 0) : 0u;
        };
        if (grp >= nS) w.item = items;
        settle();
        uint32_t step = load_steps(), parity = 0u, read_parity = 0u;
        while (w.item < items) {
            const bool is_x = w.is_x;
            const int live = min(TOK, w.c.len - blk * TOK);      // token rows of this block that belong to the chunk
            blk += (int)nS;
            settle();
            const uint32_t step_next = load_steps();
            bool ok = mbar_wait(smem_u32(&bars->full[grp]), parity, abort_flag, p.timeout_word, TO_UNPACK);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            parity ^= 1u;
            uint8_t* big = smem + (size_t)grp * stage_bytes;
            if (is_x) {
                const uint4* src = reinterpret_cast<const uint4*>(big + box * 8192 + tok * 128);
                uint4 raw[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) raw[j] = src[j ^ (tok & 7)];
                // The codes take half of the stage; expanded they take all of it, once every thread of the group has read its share.
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars->read[grp]));
                ok = mbar_wait(smem_u32(&bars->read[grp]), read_parity, abort_flag, p.timeout_word, TO_UNPACK);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                read_parity ^= 1u;
                uint8_t* out = big + box * 16384 + tok * 128;
                const bool dead = tok >= live;
#pragma unroll
                for (int j = 0; j < 8; ++j) {                    // 16 channels -> two 16-byte pieces of block j / 4 of 64 channels
                    const uint32_t s2 = step_bf16x2((step >> ((j * 16 / p.group) * 8)) & 0xFFu);
                    uint32_t v[8];
                    const uint4 w = dead ? make_uint4(0u, 0u, 0u, 0u) : raw[j];      // (and step 0: the expanded value is +0)
                    expand4(w.x, s2, v[0], v[1]);
                    expand4(w.y, s2, v[2], v[3]);
                    expand4(w.z, s2, v[4], v[5]);
                    expand4(w.w, s2, v[6], v[7]);
                    uint8_t* row = out + (j >> 2) * 8192;
                    const int c16 = (j & 3) * 2;
                    *reinterpret_cast<uint4*>(row + ((c16 ^ (tok & 7)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
                    *reinterpret_cast<uint4*>(row + (((c16 + 1) ^ (tok & 7)) << 4)) = make_uint4(v[4], v[5], v[6], v[7]);
                }
            }
            if (live < TOK) {                                    // rows of the next example: zero in the factors, and in dY
                const int from = is_x ? 4 : 0, rows = TOK - live;
                for (int i = tid; i < (4 - from + boxes) * rows * 8; i += 128) {
                    const int b = from + i / (rows * 8), rest = i % (rows * 8);
                    *reinterpret_cast<uint4*>(big + b * 8192 + (live + (rest >> 3)) * 128 + (rest & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
            }
            if (is_x || live < TOK) {
                fence_proxy_async_smem();
                __syncwarp();
            }
            if (lane == 0) mbar_arrive(smem_u32(&bars->ready[grp]));
            step = step_next;
        }
    } else {
        const int row = (warp & 3) * 32 + lane;
        const int64_t width_all = (int64_t)p.rank * (p.in + p.out);
        uint32_t n = 0;
        bool ok = true;
        Walk w;
        for (first_item(w); w.item < items && ok; next_item(w)) {
            const LoraChunk c = w.c;
            const bool is_x = w.is_x; const int ch0 = w.ch0;
            const int width = is_x ? p.in : p.out;
            for (int t0 = 0; t0 < c.len || t0 == 0; t0 += span, ++n) {
                const uint32_t buf = n & 1u;
                ok = mbar_wait(smem_u32(&bars->d_full[buf]), (n >> 1) & 1u, abort_flag, p.timeout_word, TO_EPILOGUE);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after();
                const int64_t base = is_x ? 0 : (int64_t)p.rank * p.in;
                for (int m = 0; m < 2; ++m) {
                    if (ch0 + m * 128 >= width) break;
                    const int64_t ch = ch0 + m * 128 + (warp & 3) * 32;
                    for (int c0 = 0; c0 < p.rank; c0 += 16) {
                        uint32_t v[16];
                        const uint32_t taddr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + buf * 256 + m * 128 + c0;
                        tmem_ld_x16(taddr, v);
                        tmem_wait_ld();
                        if (WIDE) {
#pragma unroll
                            for (int q = 1; q < (BOXES == 3 ? 2 : PARTS); ++q) {
                                uint32_t low[16];
                                tmem_ld_x16(taddr + (BOXES == 3 ? 64 : q * p.nr), low);
                                tmem_wait_ld();
#pragma unroll
                                for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) + __uint_as_float(low[j]));
                            }
                        }
                        if (c.len == 0) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[j] = 0u;
                        }
                        if (c.slot >= 0) store_columns(p.part + (int64_t)c.slot * width_all + base, is_x, ch, lane, width, c0, p.rank, v, PARTS == 3 && t0 > 0);
                        else store_columns(reinterpret_cast<OutT*>(p.grads) + (int64_t)c.example * p.ld_grads + base, is_x, ch, lane, width, c0, p.rank, v, PARTS == 3 && t0 > 0);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars->d_empty[buf]));
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, 512); }
}

// Adds the pieces of the examples that were summed in more than one, in piece order.
template <typename OutT>
__global__ void lora_join_kernel(const LoraJoin* __restrict__ joins, const float* __restrict__ part, int64_t width, OutT* __restrict__ grads,
                                 int64_t ld_grads)
{
    ahead_release();
    ahead_wait();
    const LoraJoin j = joins[blockIdx.y];
    for (int64_t i = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * 4; i < width; i += (int64_t)gridDim.x * blockDim.x * 4) {
        const float* src = part + (int64_t)j.first * width + i;
        float4 x = *reinterpret_cast<const float4*>(src);
        for (int k = 1; k < j.count; ++k) {
            const float4 y = *reinterpret_cast<const float4*>(src + (int64_t)k * width);
            x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
        }
        __align__(16) OutT o[4] = {to_out<OutT>(x.x), to_out<OutT>(x.y), to_out<OutT>(x.z), to_out<OutT>(x.w)};
        OutT* dst = grads + (int64_t)j.example * ld_grads + i;
        if (sizeof(OutT) == 4) *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(o);
        else *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(o);
    }
}

// Host tables reach the device as kernel arguments: no copy from pageable memory that could wait for the stream, and the call can be
// captured into a graph.
struct Words { uint64_t w[480]; };
__global__ void upload_kernel(const __grid_constant__ Words src, uint64_t* __restrict__ dst, int n)
{
    ahead_release();
    ahead_wait();
    if ((int)threadIdx.x < n) dst[threadIdx.x] = src.w[threadIdx.x];
}
cudaError_t upload(const void* host, size_t bytes, void* dev, cudaStream_t st)
{
    const size_t words = (bytes + 7) / 8;
    for (size_t w0 = 0; w0 < words; w0 += 480) {
        const size_t n = words - w0 < 480 ? words - w0 : 480;
        Words arg;
        const size_t len = bytes - w0 * 8 < n * 8 ? bytes - w0 * 8 : n * 8;
        memcpy(arg.w, reinterpret_cast<const uint8_t*>(host) + w0 * 8, len);
        const cudaError_t e = launch_ahead(upload_kernel, dim3(1), dim3(512), 0, st, arg, reinterpret_cast<uint64_t*>(dev) + w0, (int)n);
        if (e != cudaSuccess) return e;
        count_launches(1);
    }
    return cudaSuccess;
}

}  // namespace

LoraPlan plan_lora(int64_t T, int64_t n, int32_t in, int32_t out, int32_t rank, qless_dtype dtype)
{
    LoraPlan pl;
    const int64_t sms = sm_count();
    pl.nr = (rank + 15) / 16 * 16;
    pl.n64 = pl.nr <= 64 ? 64 : 128;
    pl.parts = dtype == QLESS_F32 ? 3 : 2;
    // Terms of at most 128 columns in all lie side by side; otherwise each fills its own blocks of 64 columns.
    const bool wide = pl.parts * pl.nr <= 128;
    pl.term = wide ? pl.nr : pl.n64;
    pl.boxes = wide ? (pl.parts * pl.nr + 63) / 64 : pl.parts * (pl.n64 / 64);
    pl.tiles_x = (in + TILE - 1) / TILE;
    pl.tiles = pl.tiles_x + (out + TILE - 1) / TILE;
    // Pieces of at most `chunk` tokens: about two items per SM where the examples alone do not give that many (four: 116 instead of 110 us for
    // 32 examples, 107 instead of 94 us for one of 34972 tokens: more sums to join), at least 512 tokens (a piece of fewer tokens writes
    // and re-reads more partial sums than the activations it reads).
    int64_t chunk = (T * pl.tiles + 2 * sms - 1) / (2 * sms);
    if (chunk < 512) chunk = 512;
    pl.chunk = (chunk + TOK - 1) / TOK * TOK;
    const int64_t most = T / pl.chunk;
    pl.max_slots = most + (n < most ? n : most);
    pl.max_chunks = n + most;
    pl.token_tiles = (T + 127) / 128;
    // Channel slices: about one and a half items per SM, each of at least four blocks of 128 channels (slices cost a pass that adds them).
    const int32_t kb = ((in > out ? in : out) + CH - 1) / CH;
    int64_t slices = pl.token_tiles > 0 ? (3 * sms / 2 + 2 * pl.token_tiles - 1) / (2 * pl.token_tiles) : 1;
    if (slices > (kb + 3) / 4) slices = (kb + 3) / 4;
    pl.slices = (int32_t)(slices < 1 ? 1 : slices);
    size_t off = 0;
    pl.fac_off = off; off += align_up((size_t)2 * (T > 0 ? T : 1) * pl.boxes * 128, 256);
    pl.fpart_off = off; off += align_up((size_t)2 * pl.slices * T * pl.n64 * 4, 256);
    pl.part_off = off; off += align_up((size_t)pl.max_slots * rank * ((size_t)in + out) * 4, 256);
    pl.chunk_off = off; off += align_up((size_t)pl.max_chunks * sizeof(LoraChunk), 256);
    pl.join_off = off; off += align_up((size_t)(pl.max_slots + 1) * sizeof(LoraJoin), 256);
    pl.total = off + 256;
    return pl;
}

qless_status launch_lora(const LoraArgs& a, const LoraPlan& pl, uint8_t* ws, unsigned int* timeout_word, cudaStream_t st)
{
    LoraChunk* d_chunks = reinterpret_cast<LoraChunk*>(ws + pl.chunk_off);
    LoraJoin* d_joins = reinterpret_cast<LoraJoin*>(ws + pl.join_off);
    if (a.num_chunks > INLINE) QLESS_CUDA_TRY(upload(a.chunks, (size_t)a.num_chunks * sizeof(LoraChunk), d_chunks, st));
    if (a.num_joins > 0) QLESS_CUDA_TRY(upload(a.joins, (size_t)a.num_joins * sizeof(LoraJoin), d_joins, st));
    __nv_bfloat16* fac = reinterpret_cast<__nv_bfloat16*>(ws + pl.fac_off);
    const size_t budget = 227 * 1024 - 1024 - sizeof(Bars) - 64;
    const int64_t rows = a.T > 0 ? a.T : 1;                   // no tokens at all: the maps are not used, every item has length 0
    const void* codes = a.T > 0 ? (const void*)a.codes : ws;
    const void* dy = a.T > 0 ? a.grad_out : ws;
    const int64_t ldc = a.T > 0 ? a.ld_codes : a.in, ldy = (a.T > 0 ? a.ld_grad_out : a.out) * 2;
    const bool x_whole = a.in % 128 == 0, y_whole = a.out % 64 == 0;
    const int boxes = pl.boxes;
    LoraMaps m;
    qless_status s;
    if ((s = make_tmap_2d_sw128(&m.codes1, codes, 1, a.in, rows, ldc, 128, 128)) != QLESS_OK) return s;
    if ((s = x_whole ? make_tmap_blocks_sw128(&m.codes2, codes, 1, a.in / 128, rows, ldc, 128, TOK, 2)
                     : make_tmap_2d_sw128(&m.codes2, codes, 1, a.in, rows, ldc, 128, TOK)) != QLESS_OK) return s;
    if ((s = y_whole ? make_tmap_blocks_sw128(&m.dy1, dy, 2, a.out / 64, rows, ldy, 128, 128, 2)
                     : make_tmap_2d_sw128(&m.dy1, dy, 2, a.out, rows, ldy, 64, 128)) != QLESS_OK) return s;
    if ((s = y_whole ? make_tmap_blocks_sw128(&m.dy2, dy, 2, a.out / 64, rows, ldy, 128, TOK, 4)
                     : make_tmap_2d_sw128(&m.dy2, dy, 2, a.out, rows, ldy, 64, TOK)) != QLESS_OK) return s;
    if ((s = make_tmap_2d_sw128(&m.a, a.T > 0 ? a.lora_a : ws, 2, a.in, a.rank, (uint64_t)a.in * 2, 64, pl.nr)) != QLESS_OK) return s;
    if ((s = make_tmap_2d_sw128(&m.b, a.T > 0 ? a.lora_b : ws, 2, a.rank, a.out, (uint64_t)a.rank * 2, 64, 128)) != QLESS_OK) return s;
    if ((s = make_tmap_blocks_sw128(&m.fac, fac, 2, 2 * boxes, rows, 128, rows * 128, TOK, boxes)) != QLESS_OK) return s;
    const int per = 128 / a.group;                            // step bytes of 128 channels: one load where they are one aligned word
    const bool steps_whole = reinterpret_cast<uintptr_t>(a.scales) % per == 0 && a.ld_scales % per == 0;
    if (a.T > 0) {
        FactorParams f;
        f.T = a.T; f.ld_scales = a.ld_scales; f.scales = a.scales;
        f.part = reinterpret_cast<float*>(ws + pl.fpart_off);
        f.in = a.in; f.out = a.out; f.group = a.group; f.nr = pl.nr; f.n64 = pl.n64; f.parts = pl.parts; f.term = pl.term; f.boxes = pl.boxes; f.slices = pl.slices;
        f.fac = fac; f.scaling = a.scaling;
        f.kb_x = ((a.in + CH - 1) / CH + pl.slices - 1) / pl.slices;
        f.kb_y = ((a.out + CH - 1) / CH + pl.slices - 1) / pl.slices;
        f.token_tiles = (int32_t)pl.token_tiles;
        f.items = 2 * pl.token_tiles * pl.slices;
        f.y_whole = y_whole; f.steps_whole = steps_whole;
        f.span = a.dtype == QLESS_F32 ? SPAN / CH : 1 << 24;
        f.timeout_word = timeout_word;
        const size_t stage = BIG + (size_t)pl.n64 * 256;
        f.stages = (int32_t)(budget / stage < MAX_STAGES ? budget / stage : MAX_STAGES);
        const size_t smem = 1024 + f.stages * stage + sizeof(Bars);
        const int64_t grid = f.items < sm_count() ? f.items : sm_count();
        { ProfileScope ps("lora_factors", st);
          QLESS_CUDA_TRY(allow_full_smem<lora_factors_kernel>());
          QLESS_CUDA_TRY(launch_ahead(lora_factors_kernel, dim3((unsigned)grid), dim3(NTHREADS), smem, st, m, f)); }
        if (pl.slices > 1) {
          ProfileScope ps("lora_split", st);
          const int64_t blocks = (2 * a.T * (pl.n64 / 4) + 255) / 256, most = (int64_t)sm_count() * 8;
          QLESS_CUDA_TRY(launch_ahead(lora_split_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, st, (const float*)f.part, fac, a.T, pl.n64,
                                      pl.nr, pl.slices, pl.parts, pl.term, pl.boxes, a.scaling));
          count_launches(1);
        }
        QLESS_CUDA_TRY(cudaGetLastError());
        count_launches(1);
    }
    OuterParams o;
    o.chunks = a.num_chunks > INLINE ? d_chunks : nullptr;
    if (o.chunks == nullptr) memcpy(o.few, a.chunks, (size_t)a.num_chunks * sizeof(LoraChunk)); o.scales = a.scales; o.ld_scales = a.ld_scales; o.ld_grads = a.ld_grads;
    o.grads = a.grads; o.part = reinterpret_cast<float*>(ws + pl.part_off);
    o.in = a.in; o.out = a.out; o.rank = a.rank; o.group = a.group; o.nr = pl.nr;
    o.tiles_x = pl.tiles_x; o.tiles = pl.tiles; o.timeout_word = timeout_word;
    o.x_whole = x_whole; o.y_whole = y_whole; o.steps_whole = steps_whole;
    o.items = (int64_t)a.num_chunks * pl.tiles;
    QLESS_REQUIRE(o.items < ((int64_t)1 << 31) - 65536, QLESS_ERR_UNSUPPORTED, "too many examples: %lld pieces of %d tiles", (long long)a.num_chunks, pl.tiles);
    const size_t stage = BIG + (size_t)boxes * 8192;
    o.stages = (int32_t)(budget / stage < MAX_STAGES ? budget / stage : MAX_STAGES);
    const size_t smem = 1024 + o.stages * stage + sizeof(Bars);
    const int64_t grid = o.items < sm_count() ? o.items : sm_count();
    { ProfileScope ps("lora_outer", st);
#define QLESS_LAUNCH_LORA_OUTER(OUT, N)                                                                                              \
      {                                                                                                                                \
          QLESS_CUDA_TRY((allow_full_smem<lora_outer_kernel<OUT, N>>()));                                                              \
          QLESS_CUDA_TRY(launch_ahead(lora_outer_kernel<OUT, N>, dim3((unsigned)grid), dim3(NTHREADS), smem, st, m, o));                \
      }
      if (a.dtype == QLESS_F32) {
          if (boxes == 1) QLESS_LAUNCH_LORA_OUTER(float, 1)
          else if (boxes == 2) QLESS_LAUNCH_LORA_OUTER(float, 2)
          else if (boxes == 3) QLESS_LAUNCH_LORA_OUTER(float, 3)
          else QLESS_LAUNCH_LORA_OUTER(float, 6)
      } else {
          if (boxes == 1) QLESS_LAUNCH_LORA_OUTER(__nv_bfloat16, 1)
          else if (boxes == 2) QLESS_LAUNCH_LORA_OUTER(__nv_bfloat16, 2)
          else QLESS_LAUNCH_LORA_OUTER(__nv_bfloat16, 4)
      }
#undef QLESS_LAUNCH_LORA_OUTER
    }
    QLESS_CUDA_TRY(cudaGetLastError());
    count_launches(1);
    for (int64_t j0 = 0; j0 < a.num_joins; j0 += 65535) {
        ProfileScope ps("lora_join", st);
        const int64_t width = (int64_t)a.rank * (a.in + a.out);
        const int64_t bx = (width / 4 + 255) / 256;
        const dim3 g((unsigned)(bx < 1024 ? bx : 1024), (unsigned)(a.num_joins - j0 < 65535 ? a.num_joins - j0 : 65535));
        const LoraJoin* list = d_joins + j0;
        const float* part = o.part;
        if (a.dtype == QLESS_F32) QLESS_CUDA_TRY(launch_ahead(lora_join_kernel<float>, g, dim3(256), 0, st, list, part, width, reinterpret_cast<float*>(a.grads), a.ld_grads));
        else QLESS_CUDA_TRY(launch_ahead(lora_join_kernel<__nv_bfloat16>, g, dim3(256), 0, st, list, part, width, reinterpret_cast<__nv_bfloat16*>(a.grads), a.ld_grads));
        count_launches(1);
    }
    return QLESS_OK;
}

}  // namespace qless
