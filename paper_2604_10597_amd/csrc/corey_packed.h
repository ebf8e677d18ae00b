// What the kernels on packed batches share: the layout of the index that corey_pack_plan builds, and its checks.
#ifndef COREY_PACKED_H
#define COREY_PACKED_H

#include <hip/hip_runtime.h>

#include "corey_internal.h"

namespace corey_packed {

constexpr int kMagic = 0x434f5250;
constexpr int kHead = 16;                 // words of the head: magic, S, T, tile, tokens, tiles, blocks, sequences of more than one tile
constexpr int kBlock = COREY_PACK_BLOCK;  // tokens of the small pieces

// A piece: `count` tokens of sequence `seq` from row `first` on; bits: 1 the sequence's first piece, 2 its last.
struct __align__(16) Piece {
    int32_t seq, first, count, bits;
};

// Tiles are whole blocks.
inline bool good_tile(int32_t tile) { return tile >= COREY_PACK_BLOCK && tile <= COREY_PACK_MAX_TILE && tile % COREY_PACK_BLOCK == 0; }

// Word offsets of the index's parts.
struct Layout {
    int64_t starts, seq, tiles, blocks, tile_begin, block_begin, longs, words, max_tiles, max_blocks, max_longs;
};
inline Layout layout(int64_t S, int64_t T, int32_t tile)
{
    const auto up = [](int64_t v) { return (v + 3) / 4 * 4; };      // parts begin at whole 16 bytes
    const int64_t few = S < T ? S : T;                              // a piece holds a token at least
    Layout l;
    l.max_tiles = T / tile + few;
    l.max_blocks = T / kBlock + few;
    l.starts = kHead;
    l.seq = l.starts + up(S + 1);
    l.tiles = l.seq + up(T);
    l.blocks = l.tiles + 4 * l.max_tiles;
    l.tile_begin = l.blocks + 4 * l.max_blocks;
    l.block_begin = l.tile_begin + up(S + 1);
    l.max_longs = T / (tile + 1) < S ? T / (tile + 1) : S;
    l.longs = l.block_begin + up(S + 1);
    l.words = l.longs + up(l.max_longs);
    return l;
}

// The index as the kernels take it.
struct Index {
    const int32_t* head;
    const int32_t* starts;
    const int32_t* tile_begin;            // [S + 1] the first tile of each sequence
    const int32_t* block_begin;           // [S + 1] the first block
    const int32_t* longs;                 // the sequences of more than one tile, head[7] of them
    const Piece* tiles;
    const Piece* blocks;
    int32_t S, T, tile;
    // An index of other sizes than the call was made for (memory that is no index, one that was built again) is not followed:
    // a kernel that sees one does nothing.
    __device__ __forceinline__ bool good() const { return head[0] == kMagic && head[1] == S && head[2] == T && head[3] == tile; }
};

// The checks every call on a packed batch makes; fills *ix.
inline int index_of(const char* who, const corey_pack* p, Index* ix)
{
    using corey::fail;
    if (!p || !p->table) return fail(COREY_ENULL, "%s: the index is NULL (corey_pack_plan fills it)", who);
    if (p->S < 1 || p->T < 1 || p->T > INT32_MAX || p->S > COREY_PACK_MAX_SEQS || !good_tile(p->tile))
        return fail(COREY_EINVAL, "%s: the index was not filled by corey_pack_plan", who);
    const Layout l = layout(p->S, p->T, p->tile);
    if (p->bytes < (size_t)l.words * 4 || reinterpret_cast<uintptr_t>(p->table) % 16 != 0)
        return fail(COREY_EWORKSPACE, "%s: the index's memory is too small or not 16-byte aligned", who);
    const int32_t* w = static_cast<const int32_t*>(p->table);
    ix->head = w;
    ix->starts = w + l.starts;
    ix->tile_begin = w + l.tile_begin;
    ix->block_begin = w + l.block_begin;
    ix->longs = w + l.longs;
    ix->tiles = reinterpret_cast<const Piece*>(w + l.tiles);
    ix->blocks = reinterpret_cast<const Piece*>(w + l.blocks);
    ix->S = (int32_t)p->S;
    ix->T = (int32_t)p->T;
    ix->tile = p->tile;
    return COREY_OK;
}

// The slot a sequence's state is read from (or left in); -1: none.
__device__ __forceinline__ int64_t slot_of(const int32_t* slots, int seq, int64_t n_slots)
{
    if (!slots) return -1;
    const int32_t s = slots[seq];
    return s >= 0 && s < n_slots ? s : -1;
}

// Rows of `stride` elements between tokens: at least D, and 15 of them stay below 2^31 bytes of the widest type.
constexpr int64_t kMaxStride = (int64_t)1 << 25;
inline bool good_stride(int64_t stride, int64_t D) { return stride >= D && stride < kMaxStride; }

// A launch has fewer than 2^32 lanes.
inline bool good_grid(int64_t groups, int64_t threads) { return groups * threads <= UINT32_MAX; }

inline bool good_dtype(corey_dtype dt) { return dt == COREY_F32 || dt == COREY_BF16 || dt == COREY_F16; }

// f(T()) with the storage type of dt.
template <typename F> inline void by_type(corey_dtype dt, F&& f)
{
    if (dt == COREY_F32) f(float());
    else if (dt == COREY_F16) f(_Float16());
    else f(uint16_t());
}

}  // namespace corey_packed
#endif
