// What the forward and backward scans of packed batches share: their arguments, B and C in scalar registers, the loads of a block
// of tokens.
#ifndef COREY_PACKED_SCAN_H
#define COREY_PACKED_SCAN_H

#include <hip/hip_runtime.h>

#include "corey_packed.h"
#include "corey_scan_impl.h"

namespace corey_packed {

using corey_scan::exp2_burst;
using corey_scan::fast_exp2;
using corey_scan::Io;
using corey_scan::kLn2;
using corey_scan::kLog2e;
using corey_scan::rcp_burst;
using corey_scan::silu;
using corey_scan::softplus;

constexpr int kStates = 16;               // states of a wave; more are more waves of one workgroup

struct PackedScanArgs {
    Index ix;
    const void *u, *delta, *Bm, *Cm, *z;
    const float *A, *Dv, *bias;
    void* y;
    float* state;                         // [n_slots, D, N]
    const int32_t *slots, *slots_out;
    int64_t u_stride, d_stride, b_stride, c_stride, z_stride, y_stride, n_slots;
    float* bc;                            // workspace [blocks, 2 halves, N, (B, C), 8 tokens]
    float* ends;                          // workspace [tiles, N, D]: a tile's end state from zero, then the state it begins with
    float* sums;                          // workspace [tiles, D]: a tile's sum of step sizes
    int32_t D, N, groups, softplus;       // groups: of channels, one per workgroup
    int32_t blocks;
    // backward
    const void* dy;
    void *du, *ddelta, *dz, *dB, *dC;
    float *dA, *dD, *dbias;
    int64_t dy_stride, du_stride, dd_stride, dz_stride, db_stride, dc_stride;
    float* backs;                         // workspace [tiles, N, D]: what a tile hands to the gradient of the state it begins with
    float* starts;                        // workspace [tiles, tile / 16 - 1, N, D]: the states that a tile's blocks 1, 2, ... begin with when
                                          // the tile begins from zero
    float* start_sums;                    // workspace [tiles, tile / 16 - 1, D]: the sums of the step sizes before them
    float* part_bc;                       // workspace [channel groups, blocks, N, 16 tokens, (dB, dC)]
    float* part_a;                        // workspace [tiles, N + 2, D]: dA, dD and dbias of a tile
};

// B and C are the same for every channel: a wave takes them into scalar registers, where they are operands like any other and cost
// neither vector registers nor LDS.  Scalar loads want them as binary32 and in the order of use, so a launch in front writes them
// so: per block of 16 tokens, half of it and state, B of the 8 tokens and then C (zeros behind the block's last token).
constexpr int kHalf = 8;
template <typename T> __global__ __launch_bounds__(256) void k_packed_relay(PackedScanArgs a)
{
    const int per = 4 * kHalf * a.N;                             // values of a block
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t block = i / per;
    if (block >= a.blocks || !a.ix.good()) return;
    const Piece p = a.ix.blocks[block];
    if (p.seq < 0) return;
    const int j = (int)(i - block * per), half = j / (2 * kHalf * a.N), c = (j >> 3) & 1, n = (j >> 4) - half * a.N;
    const int t = half * kHalf + (j & (kHalf - 1));
    const T* row = c ? static_cast<const T*>(a.Cm) + (p.first + (int64_t)t) * a.c_stride : static_cast<const T*>(a.Bm) + (p.first + (int64_t)t) * a.b_stride;
    a.bc[i] = t < p.count ? Io<T>::ld(row + n) : 0.f;
}

// B and C of one state for 8 tokens, from memory that no kernel writes while this one runs, at a place that is the same for the whole
// wave.
struct State8 {
    typedef float Vec __attribute__((ext_vector_type(2 * kHalf)));
    Vec v;
    __device__ __forceinline__ float b(int t) const { return v[t]; }
    __device__ __forceinline__ float c(int t) const { return v[kHalf + t]; }
};
__device__ __forceinline__ State8 state8(const float* p)
{
    State8 s;
    s.v = *(const __attribute__((address_space(4))) State8::Vec*)(uintptr_t)p;
    return s;
}

// States n and n + 1 of a wave, and the two behind them on their way: scalar loads come back in any order, so a wait for one is a wait
// for all, and each pair is asked for two states of work ahead.
struct StatePairs {
    State8 s[2][2];
    const float* from;
    __device__ __forceinline__ explicit StatePairs(const float* p) : from(p)
    {
        s[0][0] = state8(from);
        s[0][1] = state8(from + 2 * kHalf);
    }
    __device__ __forceinline__ const State8& at(int n) const { return s[(n >> 1) & 1][n & 1]; }
    // at the start of state n's work (behind the wave's last states: the next block's, or the workspace's end)
    __device__ __forceinline__ void ahead(int n)
    {
        if ((n & 1) != 0 || n + 2 >= kStates) return;
        s[((n >> 1) + 1) & 1][0] = state8(from + (n + 2) * 2 * kHalf);
        s[((n >> 1) + 1) & 1][1] = state8(from + (n + 3) * 2 * kHalf);
    }
};

// The blocks a tile's tokens lie in: the number of the first.
__device__ __forceinline__ int64_t first_block(const Index& ix, const Piece& p) { return ix.block_begin[p.seq] + (p.first - ix.starts[p.seq]) / kBlock; }

// The rows of one tensor from some token on: a wave's address is a scalar row and each lane's place in it (`off`, in bytes).  Written
// with the buffer instructions, which take both as they are (left to plain pointers the compiler adds them per lane, in 64 bits).
template <typename T> struct Rows {
    const char* first;                                           // the row of the first token
    uint32_t step;                                               // bytes from row to row: 15 steps fit 31 bits (kMaxStride)
    __device__ __forceinline__ Rows(const void* base, int64_t stride, int64_t token)
        : first(static_cast<const char*>(base) + token * stride * (int64_t)sizeof(T)), step((uint32_t)stride * (uint32_t)sizeof(T))
    {
    }
    __device__ __forceinline__ void advance(int tokens) { first += (int64_t)tokens * step; }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t resource() const
    {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(first), 0, 0xffffffffu, 0x00020000);
    }
};

// C tokens of one channel, as stored.  Of them `count` >= 1 are there; the others' rows are replaced by the last one's.
template <typename T, int C> struct Tokens {
    T v[C];
    __device__ __forceinline__ float at(int t) const { return Io<T>::ld(&v[t]); }
};
template <typename T, int C> __device__ __forceinline__ Tokens<T, C> load_tokens(const Rows<T>& rows, int count, uint32_t off)
{
    Tokens<T, C> k;
    const auto r = rows.resource();
#pragma unroll
    for (int t = 0; t < C; ++t) {
        const uint32_t row = (uint32_t)min(t, count - 1) * rows.step;
        if constexpr (sizeof(T) == 2) {
            const uint16_t v = __builtin_amdgcn_raw_buffer_load_b16(r, off, row, 0);
            __builtin_memcpy(&k.v[t], &v, 2);
        } else {
            const uint32_t v = __builtin_amdgcn_raw_buffer_load_b32(r, off, row, 0);
            __builtin_memcpy(&k.v[t], &v, 4);
        }
    }
    return k;
}

// C results of one channel, rounded to T; the first `count` of them are stored.
template <typename T, int C> __device__ __forceinline__ void store_tokens(const Rows<T>& rows, int count, uint32_t off, const float (&v)[C])
{
    const auto r = rows.resource();
    const auto put = [&](int t, float x, float y, bool second) {
        if constexpr (sizeof(T) == 2) {
            const uint32_t w = Io<T>::pack2(x, y);
            __builtin_amdgcn_raw_buffer_store_b16((uint16_t)w, r, off, (uint32_t)t * rows.step, 0);
            if (second) __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(w >> 16), r, off, (uint32_t)(t + 1) * rows.step, 0);
        } else {
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), r, off, (uint32_t)t * rows.step, 0);
            if (second) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(y), r, off, (uint32_t)(t + 1) * rows.step, 0);
        }
    };
    if (count >= C) {
#pragma unroll
        for (int t = 0; t < C; t += 2) put(t, v[t], v[t + 1], true);
    } else {
#pragma unroll
        for (int t = 0; t < C; t += 2)
            if (t < count) put(t, v[t], v[t + 1], t + 1 < count);
    }
}

// Step sizes and their products with u; tokens behind the piece get 0 for both: the state stays as it is (and a NaN among the
// replaced rows stays out).
template <typename T, int C>
__device__ __forceinline__ void steps(const Tokens<T, C>& u, const Tokens<T, C>& delta, float bias, bool sp, int count, float (&dl)[C], float (&dx)[C])
{
#pragma unroll
    for (int t = 0; t < C; ++t) dl[t] = delta.at(t) + bias;
    if (sp) corey_scan::softplus_all<C>(dl);
#pragma unroll
    for (int t = 0; t < C; ++t) dx[t] = dl[t] * u.at(t);
    if (count < C) {
#pragma unroll
        for (int t = 0; t < C; ++t) {
            dl[t] = t < count ? dl[t] : 0.f;
            dx[t] = t < count ? dx[t] : 0.f;
        }
    }
}

// silu(z) of C tokens
template <typename T, int C> __device__ __forceinline__ void gates(const Tokens<T, C>& z, float (&g)[C])
{
#pragma unroll
    for (int t = 0; t < C; ++t) g[t] = -z.at(t) * kLog2e;
    exp2_burst<C>(g);
#pragma unroll
    for (int t = 0; t < C; ++t) g[t] += 1.f;
    rcp_burst<C>(g);
#pragma unroll
    for (int t = 0; t < C; ++t) g[t] *= z.at(t);
}

// The arguments of C decays and the products dx B, one after the other.  An instruction that reads a scalar register issues beside one
// of another wave that reads none, but not beside one that does: the products (which read B from scalar registers) and the arguments
// alternate, and so do, behind the exponentials, the states' updates and the sums (which read C).  Cycles of a SIMD for a wave's state
// and 8 tokens, four waves: products behind the exponentials, with the updates and sums, 171; alternating 148; 128 if all paired.
template <int C, typename F> __device__ __forceinline__ void arguments(const float (&dl)[C], float a2, const float (&dx)[C], F&& b, float (&e)[C], float (&p)[C])
{
#pragma unroll
    for (int t = 0; t < C; ++t) {
        e[t] = dl[t] * a2;
        p[t] = dx[t] * b(t);
    }
#pragma unroll
    for (int t = 0; t < C; ++t) asm volatile("" : "+v"(p[t]));
    exp2_burst<C>(e);
}

// A for decays in base 2.  Where the product leaves binary32 it stays a number: a step size of 0 (of tokens that are not there) times it
// is 0, and any other's decay is 0 as well.
__device__ __forceinline__ float rate(float a)
{
    const float r = a * kLog2e;
    return r == -__builtin_huge_valf() ? -__FLT_MAX__ : r;
}

// States n0 .. n0 + C - 1 of a row of N in memory; 0 at and behind N.
template <int C> __device__ __forceinline__ void load_row(float (&out)[C], const float* row, int n0, int N)
{
#pragma unroll
    for (int n = 0; n < C; ++n) out[n] = 0.f;
    if (N % 4 == 0) {                     // whole groups of four: one load each, at any alignment
#pragma unroll
        for (int n = 0; n < C; n += 4)
            if (n0 + n < N) __builtin_memcpy(&out[n], row + n, 16);
    } else {
#pragma unroll
        for (int n = 0; n < C; ++n)
            if (n0 + n < N) out[n] = row[n];
    }
}

// A workgroup's waves are 64 channels each with all states, up to 16 states (CHANNEL_WAVES of them: they read the same B and C, from
// the scalar cache of their compute unit after the first), or 64 channels between them with 16 states each.
constexpr int kChannelWaves = 4;
template <int GROUPS> struct Shape {
    static constexpr int channel_waves = GROUPS == 1 ? kChannelWaves : 1, waves = GROUPS * channel_waves, channels = 64 * channel_waves;
};
inline int64_t channel_groups(int64_t D, int64_t N) { return N <= kStates ? (D + 64 * kChannelWaves - 1) / (64 * kChannelWaves) : (D + 63) / 64; }

// f(GROUPS): the waves that share a channel's states, 16 each.
template <typename F> void by_groups(int64_t N, F&& f)
{
    if (N <= 16) f(std::integral_constant<int, 1>());
    else if (N <= 32) f(std::integral_constant<int, 2>());
    else if (N <= 64) f(std::integral_constant<int, 4>());
    else f(std::integral_constant<int, 8>());
    static_assert(COREY_PACK_MAX_STATE == 8 * kStates, "the widest workgroup holds all states");
}
inline int64_t waves_of(int64_t N)        // of a workgroup
{
    int64_t waves = 0;
    by_groups(N, [&](auto g) { waves = Shape<decltype(g)::value>::waves; });
    return waves;
}

}  // namespace corey_packed
#endif
