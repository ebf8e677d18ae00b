// corey_pack_plan: the index of a packed batch from the lengths of its sequences.
//
//   starts[s] = min(T, sum of the lengths before s)      (lengths below 0 count as 0; what does not fit into T rows is cut off)
//   seq[t]    = the sequence whose [starts[s], starts[s+1]) holds t, -1 behind the last
//   tiles     = every sequence cut into pieces of `tile` tokens, in order; blocks: into pieces of 16
//
// Nothing but latency bounds it (a few MB at most).  Up to kOneLaunch sequences every workgroup sums the lengths up for itself in
// LDS and fills its own part of the maps from them: one launch, no workgroup waits for another.  Beyond that one workgroup
// sums and a second launch fills.  Adding with a cap, min(T, a + b), is associative for values of 0 .. T, so the cut rows
// need no pass of their own, and no sum leaves 32 bits.
#include <hip/hip_runtime.h>

#include "corey_packed.h"

namespace {

using namespace corey_packed;

constexpr int kThreads = 512;
constexpr int kWavesPer = kThreads / 64;
constexpr int kOneLaunch = 4096;          // three prefix sums of 16 KB each in LDS
constexpr int kRun = kOneLaunch / kThreads;   // sequences of a lane
constexpr int kPer = 4;                   // tokens of a lane: one 16-byte store

struct PlanArgs {
    const int32_t* lengths;
    int32_t *head, *starts, *seq, *tile_begin, *block_begin, *longs;
    Piece *tiles, *blocks;
    int32_t S, T, tile;
    int32_t max_tiles, max_blocks;
    int32_t token_groups, tile_groups;    // workgroups for the tokens, for the tiles; the rest are for the blocks
};

__device__ __forceinline__ uint32_t add_capped(uint32_t a, uint32_t b, uint32_t cap)
{
    const uint32_t s = a + b;             // both at most 2^31 - 1
    return s < cap ? s : cap;
}

// Exclusive sums of several counts over the workgroup's lanes, each capped, and the sums of all; `scratch` has a word per wave and count.
template <int C> __device__ void scan_lanes(uint32_t (&v)[C], const uint32_t (&cap)[C], uint32_t (*scratch)[kWavesPer], uint32_t (&all)[C])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t up[C];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const uint32_t o = __shfl_up(v[c], d);
            if (lane >= d) v[c] = add_capped(v[c], o, cap[c]);
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if (lane == 63) scratch[c][wave] = v[c];
        up[c] = __shfl_up(v[c], 1);
        if (lane == 0) up[c] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < C; ++c) {
        uint32_t before = 0;
        all[c] = 0;
#pragma unroll
        for (int w = 0; w < kWavesPer; ++w) {
            if (w == wave) before = all[c];
            all[c] = add_capped(all[c], scratch[c][w], cap[c]);
        }
        v[c] = add_capped(before, up[c], cap[c]);
    }
    __syncthreads();
}

struct Sums {
    uint32_t tokens, tiles, blocks, longs;
};

// Exclusive sums of the tokens, tiles and blocks of n <= kOneLaunch sequences, behind `before`, into three arrays of n + 1, and
// the list of the sequences of more than one tile (where `longs` is given; s0: the first one's number).  A lane takes kRun sequences
// in a row, all of their lengths in one trip to memory.  Returns the sums behind the last.
__device__ Sums sum_up(const PlanArgs& a, int s0, int n, Sums before, int32_t* starts, int32_t* tile_begin, int32_t* block_begin,
                       int32_t* longs, uint32_t (*scratch)[kWavesPer])
{
    const uint32_t cap = (uint32_t)a.T;
    const int first = (int)threadIdx.x * kRun;
    const int32_t* lengths = a.lengths + s0;
    uint32_t len[kRun], sum[1] = {}, all[1];
#pragma unroll
    for (int i = 0; i < kRun; ++i) len[i] = first + i < n ? (uint32_t)min(max(lengths[first + i], 0), a.T) : 0u;
#pragma unroll
    for (int i = 0; i < kRun; ++i) sum[0] = add_capped(sum[0], len[i], cap);
    scan_lanes<1>(sum, {cap}, scratch, all);
    uint32_t at = add_capped(before.tokens, sum[0], cap);
    uint32_t pieces[3] = {}, of_all[3];                         // tiles, blocks, sequences of more than one tile
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        const uint32_t next = add_capped(at, len[i], cap);
        if (first + i < n) starts[first + i] = (int32_t)at;
        len[i] = next - at;                                     // what of it fits
        pieces[0] += (len[i] + a.tile - 1) / (uint32_t)a.tile;
        pieces[1] += (len[i] + kBlock - 1) / kBlock;
        pieces[2] += len[i] > (uint32_t)a.tile;
        at = next;
    }
    const uint32_t none = 0x7fffffffu;
    scan_lanes<3>(pieces, {none, none, none}, scratch, of_all);
    Sums out;
    out.tokens = add_capped(before.tokens, all[0], cap);
    out.tiles = before.tiles + of_all[0];
    out.blocks = before.blocks + of_all[1];
    out.longs = before.longs + of_all[2];
    uint32_t tb = before.tiles + pieces[0], bb = before.blocks + pieces[1], lb = before.longs + pieces[2];
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        if (first + i < n) {
            tile_begin[first + i] = (int32_t)tb;
            block_begin[first + i] = (int32_t)bb;
            if (len[i] > (uint32_t)a.tile) {
                if (longs) longs[lb] = s0 + first + i;
                ++lb;
            }
        }
        tb += (len[i] + a.tile - 1) / (uint32_t)a.tile;
        bb += (len[i] + kBlock - 1) / kBlock;
    }
    if (threadIdx.x == 0) {
        starts[n] = (int32_t)out.tokens;
        tile_begin[n] = (int32_t)out.tiles;
        block_begin[n] = (int32_t)out.blocks;
    }
    __syncthreads();
    return out;
}

// The last s with begin[s] <= i; with i < begin[S] it is the sequence that holds i.
__device__ __forceinline__ int holder(const int32_t* begin, int S, int i)
{
    int lo = 0, hi = S;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (begin[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int highest(int v) { return v > 0 ? 1 << (31 - __clz(v)) : 0; }    // the highest power of two in it

__device__ void fill_pieces(const int32_t* starts, const int32_t* begin, int S, int size, Piece* out, int i, int room)
{
    if (i >= room) return;
    Piece p{-1, 0, 0, 0};
    if (i < begin[S]) {
        const int s = holder(begin, S, i), k = i - begin[s];
        const int n = starts[s + 1] - starts[s], at = k * size;
        p.seq = s;
        p.first = starts[s] + at;
        p.count = min(n - at, size);
        p.bits = (k == 0 ? 1 : 0) + (i + 1 == begin[s + 1] ? 2 : 0);
    }
    out[i] = p;
}

__device__ void fill(const PlanArgs& a, const int32_t* starts, const int32_t* tile_begin, const int32_t* block_begin)
{
    int g = blockIdx.x;
    if (g < a.token_groups) {
        const int64_t t0 = ((int64_t)g * kThreads + threadIdx.x) * kPer;
        if (t0 >= a.T) return;
        const int used = starts[a.S];
        // Searches for the lane's first and last token side by side, then for those between them between the two: sequences without
        // tokens may be any number there (passed one by one 131072 of them took 9 ms).
        int v[kPer] = {};
        for (int step = highest(a.S - 1); step > 0; step >>= 1) {
#pragma unroll
            for (int i = 0; i < kPer; i += kPer - 1) {
                const int s = min(v[i] + step, a.S - 1);
                if (starts[s] <= t0 + i) v[i] = s;
            }
        }
#pragma unroll
        for (int i = 1; i < kPer - 1; ++i) v[i] = v[0];
        for (int step = highest(v[kPer - 1] - v[0]); step > 0; step >>= 1) {
#pragma unroll
            for (int i = 1; i < kPer - 1; ++i) {
                const int s = min(v[i] + step, v[kPer - 1]);
                if (starts[s] <= t0 + i) v[i] = s;
            }
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (t0 + i >= used) v[i] = -1;
        if (t0 + kPer <= a.T) {
            *reinterpret_cast<int4*>(a.seq + t0) = make_int4(v[0], v[1], v[2], v[3]);
        } else {
            for (int i = 0; t0 + i < a.T; ++i) a.seq[t0 + i] = v[i];
        }
        return;
    }
    g -= a.token_groups;
    if (g < a.tile_groups) fill_pieces(starts, tile_begin, a.S, a.tile, a.tiles, g * kThreads + (int)threadIdx.x, a.max_tiles);
    else fill_pieces(starts, block_begin, a.S, kBlock, a.blocks, (g - a.tile_groups) * kThreads + (int)threadIdx.x, a.max_blocks);
}

__device__ void write_head(const PlanArgs& a, const Sums& all)
{
    if (threadIdx.x < kHead) {
        const int v[8] = {kMagic, a.S, a.T, a.tile, (int)all.tokens, (int)all.tiles, (int)all.blocks, (int)all.longs};
        int w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w = (int)threadIdx.x == i ? v[i] : w;
        a.head[threadIdx.x] = w;
    }
}

__global__ __launch_bounds__(kThreads) void k_pack_small(PlanArgs a)
{
    __shared__ int32_t s_starts[kOneLaunch + 1], s_tiles[kOneLaunch + 1], s_blocks[kOneLaunch + 1];
    __shared__ uint32_t scratch[3][kWavesPer];
    const Sums all = sum_up(a, 0, a.S, Sums{0, 0, 0, 0}, s_starts, s_tiles, s_blocks, blockIdx.x == 0 ? a.longs : nullptr, scratch);
    if (blockIdx.x == 0) {
        for (int s = threadIdx.x; s <= a.S; s += kThreads) {
            a.starts[s] = s_starts[s];
            a.tile_begin[s] = s_tiles[s];
            a.block_begin[s] = s_blocks[s];
        }
        write_head(a, all);
    }
    fill(a, s_starts, s_tiles, s_blocks);
}

__global__ __launch_bounds__(kThreads) void k_pack_sums(PlanArgs a)
{
    __shared__ uint32_t scratch[3][kWavesPer];
    Sums at{0, 0, 0, 0};
    for (int s = 0; s < a.S; s += kOneLaunch)                   // (the next part overwrites this one's end with the same value)
        at = sum_up(a, s, min(kOneLaunch, a.S - s), at, a.starts + s, a.tile_begin + s, a.block_begin + s, a.longs, scratch);
    write_head(a, at);
}

__global__ __launch_bounds__(kThreads) void k_pack_fill(PlanArgs a) { fill(a, a.starts, a.tile_begin, a.block_begin); }

}  // namespace

extern "C" size_t corey_pack_bytes(int64_t S, int64_t T, int32_t tile)
{
    if (S < 1 || S > COREY_PACK_MAX_SEQS || T < 1 || T > INT32_MAX || !good_tile(tile))
        return 0;
    return (size_t)layout(S, T, tile).words * 4;
}

extern "C" int corey_pack_plan(const int32_t* lengths, int64_t S, int64_t T, int32_t tile, void* table, size_t table_bytes,
                               corey_pack* pack, void* hip_stream)
{
    using corey::fail;
    if (!lengths || !table || !pack) return fail(COREY_ENULL, "corey_pack_plan: lengths, table and pack are required");
    if (S < 1 || S > COREY_PACK_MAX_SEQS) return fail(COREY_ESHAPE, "corey_pack_plan: 1 <= S <= %d required", COREY_PACK_MAX_SEQS);
    if (T < 1 || T > INT32_MAX) return fail(COREY_ESHAPE, "corey_pack_plan: 1 <= T < 2^31 required");
    if (!good_tile(tile))
        return fail(COREY_EINVAL, "corey_pack_plan: tile must be a multiple of %d up to %d", COREY_PACK_BLOCK, COREY_PACK_MAX_TILE);
    const Layout l = layout(S, T, tile);
    if (table_bytes < (size_t)l.words * 4 || reinterpret_cast<uintptr_t>(table) % 16 != 0)
        return fail(COREY_EWORKSPACE, "corey_pack_plan: table must be 16-byte aligned and have corey_pack_bytes() bytes");
    int32_t* w = static_cast<int32_t*>(table);
    PlanArgs a;
    a.lengths = lengths;
    a.head = w;
    a.starts = w + l.starts;
    a.seq = w + l.seq;
    a.tiles = reinterpret_cast<Piece*>(w + l.tiles);
    a.blocks = reinterpret_cast<Piece*>(w + l.blocks);
    a.tile_begin = w + l.tile_begin;
    a.block_begin = w + l.block_begin;
    a.longs = w + l.longs;
    a.S = (int32_t)S;
    a.T = (int32_t)T;
    a.tile = tile;
    a.max_tiles = (int32_t)l.max_tiles;
    a.max_blocks = (int32_t)l.max_blocks;
    const auto groups = [](int64_t n, int64_t per) { return (int32_t)((n + per - 1) / per); };
    a.token_groups = groups(T, (int64_t)kThreads * kPer);
    a.tile_groups = groups(l.max_tiles, kThreads);
    const unsigned all = (unsigned)(a.token_groups + a.tile_groups + groups(l.max_blocks, kThreads));
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (S <= kOneLaunch) {
        k_pack_small<<<all, kThreads, 0, stream>>>(a);
    } else {
        k_pack_sums<<<1, kThreads, 0, stream>>>(a);
        k_pack_fill<<<all, kThreads, 0, stream>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return corey::hip_fail(e, "corey_pack_plan launch");
    pack->table = table;
    pack->bytes = table_bytes;
    pack->S = S;
    pack->T = T;
    pack->tile = tile;
    pack->reserved = 0;
    return COREY_OK;
}
