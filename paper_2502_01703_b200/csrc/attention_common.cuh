// What the attention kernels share: tiles of query rows, the table of work, small arithmetic.
//
// Query heads that read the same key head are packed into a tile's rows: with `pack` of them (the largest power of two that divides the group,
// at most 16) a tile of 128 rows holds 128 / pack tokens, row r = token r / pack, head r % pack. One copy of a three-dimensional box
// brings it, keys and values are read once for all of them, and short sequences fill their tiles better.
#pragma once

#include <functional>
#include <vector>

#include "pairs.cuh"
#include "qless_kernels.h"
#include "tc_common.cuh"

namespace qless {
namespace attn {

using namespace tc;

constexpr int TILE = 128;                   // rows of a tile of queries, and of keys
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int INLINE = 160;                 // tiles that travel in the launch itself

struct TileTable {
    const AttnTile* list;                   // NULL: few
    int32_t tiles;
    AttnTile few[INLINE];
};

__device__ __forceinline__ AttnTile tile_of(const TileTable& t, uint32_t i) { return t.list != nullptr ? t.list[i] : t.few[i]; }
__device__ __forceinline__ AttnTile uniform_tile(const AttnTile& x) { return {warp_uniform(x.t0), warp_uniform(x.len), warp_uniform(x.at), warp_uniform(x.way)}; }

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint64_t ex2_pair(uint64_t x)
{
    float a, b;
    split_pair(x, a, b);
    return pair_of(ex2(a), ex2(b));
}
__device__ __forceinline__ uint32_t pack_pair(uint64_t x)
{
    float a, b;
    split_pair(x, a, b);
    const __nv_bfloat162 z = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&z);
}
__device__ __forceinline__ float max3(float a, float b, float c)      // NaN where one of them is
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
constexpr int64_t MOST_ITEMS = (int64_t)1 << 31;      // of a launch: counted in 32 bits
// The block's item of round k: forwards and backwards in turn, so that the lists, which begin with the longest, come out even.
__device__ __forceinline__ uint32_t item_of_round(uint32_t k) { return k * gridDim.x + ((k & 1u) ? gridDim.x - 1 - blockIdx.x : blockIdx.x); }
// A role's way over the block's items (item = tile * per_tile + sub). The table's entry of the item after is read while this one is worked on.
struct Walk {
    const TileTable& table;
    uint32_t items, per_tile, round = 0, item, sub = 0;
    AttnTile tile, after;
    bool more;
    __device__ __forceinline__ Walk(const TileTable& t, uint32_t n, uint32_t per) : table(t), items(n), per_tile(per)
    {
        item = item_of_round(0);
        more = item < items;
        tile = after = AttnTile{0, 0, 0, 0};
        if (more) { after = tile_of(table, item / per_tile); arrive(); }
    }
    __device__ __forceinline__ void arrive()
    {
        sub = item - item / per_tile * per_tile;
        tile = uniform_tile(after);
        const uint32_t next = item_of_round(round + 1);
        if (next < items) after = tile_of(table, next / per_tile);
    }
    __device__ __forceinline__ void next()
    {
        item = item_of_round(++round);
        more = item < items;
        if (more) arrive();
    }
};

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const __nv_bfloat162 z = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&z);
}
__device__ __forceinline__ void unpack_bf16(const uint4& u, float (&v)[8])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { v[2 * k] = __uint_as_float(w[k] << 16); v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u); }
}

struct Ring {
    uint32_t slot = 0, parity = 0;
    __device__ __forceinline__ void next(uint32_t n) { if (++slot == n) { slot = 0; parity ^= 1u; } }
};

// Rows [from, 128) of an operand of `blocks` 64-column blocks (128 rows of 128 bytes each) become zero: by a whole warp, between the copy's
// arrival and the tensor core's reading. Rows behind a sequence's end are another sequence's (or nobody's): a zero factor alone would let
// their infinities and NaN through.
__device__ __forceinline__ void zero_rows(uint8_t* operand, int blocks, int from, int lane)
{
    for (int b = 0; b < blocks; ++b)
        for (int i = from * 8 + lane; i < TILE * 8; i += 32) *reinterpret_cast<uint4*>(operand + b * 16384 + i * 16) = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async_smem();
    __syncwarp();
}

// Rows of D bf16 values, 32 of them (columns c0 ..) in each lane for a row of its own, go to memory 64 bytes at a time: `dst` are the addresses of rows
// (lane & ~3) + 0 .. 3 of the warp's 32, NULL for one that is not written.
__device__ __forceinline__ void store_rows32(const float (&v)[32], int c0, int head_dim, int lane, __nv_bfloat16* const (&dst)[4])
{
    uint4 w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
        w[k] = make_uint4(pack_bf16(v[8 * k], v[8 * k + 1]), pack_bf16(v[8 * k + 2], v[8 * k + 3]), pack_bf16(v[8 * k + 4], v[8 * k + 5]),
                          pack_bf16(v[8 * k + 6], v[8 * k + 7]));
    transpose4(w, lane);
    const int c = c0 + (lane & 3) * 8;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (dst[k] != nullptr && c < head_dim) *reinterpret_cast<uint4*>(dst[k] + c) = w[k];
}

// Work of one launch: query tiles of `rows` tokens, or key tiles of 128, of every sequence, those with the longest loops first.
std::vector<AttnTile> query_tiles(const AttnArgs& a, int32_t tokens_per_tile);
std::vector<AttnTile> key_tiles(const AttnArgs& a);
// Fills the table, through device memory at `dev` where it does not fit into the launch.
size_t tiles_bytes(int64_t tokens, int64_t n, int64_t rows);
// Few tiles and long loops: a tile's loop is dealt out in pieces, in one round of the SMs or two, where that takes at least so many steps off the longest
// block's work, and at least three in twenty (about what the launch of the join, the join and the host's part of them cost; backward there are two, with two sums
// of a row each). Forward: 1000 tokens, 8/2 heads of 128, five steps less: 26 -> 34 us; 4000, 4/4 heads, twelve less: 63 -> 54 us; 3000, 2/1 heads, 21 less: 47 -> 27 us.
// Backward: 4000 tokens, 4/4 heads, twelve less: 116 -> 122 us; 800, 8/2 heads, 22 less: 65 -> 50 us; 3000, 2/1 heads, 21 less: 123 -> 63 us; 3000, 32/1 heads:
// 1276 -> 274 us (24 tiles of keys with up to 750 steps).
constexpr int32_t SPLIT_FORWARD = 10, SPLIT_BACKWARD = 16, SPLIT_ROUNDS = 2;
size_t split_bytes(int64_t tokens, int32_t heads, int32_t kv_heads, bool backward);
int32_t split_tiles(std::vector<AttnTile>* tiles, int32_t per, int32_t gain, const std::function<int32_t(const AttnTile&)>& loops);
qless_status put_table(const std::vector<AttnTile>& tiles, TileTable* table, AttnTile* dev, cudaStream_t st);
// [tokens][heads][head_dim] bf16, boxes of 64 columns x box_heads x box_tokens, zeros behind head_dim.
qless_status head_map(CUtensorMap* out, const void* base, int64_t ld, int32_t heads, int32_t head_dim, int64_t tokens, uint32_t box_heads, uint32_t box_tokens);

}  // namespace attn
}  // namespace qless
