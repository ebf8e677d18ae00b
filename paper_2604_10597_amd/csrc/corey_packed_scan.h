// What the forward and backward scans of packed batches share: their arguments and the loads of a block of tokens.
#ifndef COREY_PACKED_SCAN_H
#define COREY_PACKED_SCAN_H

#include <hip/hip_runtime.h>

#include "corey_packed.h"
#include "corey_scan_impl.h"

namespace corey_packed {

using corey_scan::exp2_burst;
using corey_scan::fast_exp2;
using corey_scan::float4v;
using corey_scan::Io;
using corey_scan::kLn2;
using corey_scan::kLog2e;
using corey_scan::silu;
using corey_scan::softplus;

constexpr int kStates = 16;               // states a wave keeps in registers; more are more waves of one workgroup

struct PackedScanArgs {
    Index ix;
    const void *u, *delta, *Bm, *Cm, *z;
    const float *A, *Dv, *bias;
    void* y;
    float* state;                         // [n_slots, D, N]
    const int32_t *slots, *slots_out;
    int64_t u_stride, d_stride, b_stride, c_stride, z_stride, y_stride, n_slots;
    float *ends;                          // workspace [tiles, N, D]: a tile's end state from zero, then the state it begins with
    float *sums;                          // workspace [tiles, D]: a tile's sum of step sizes
    int32_t D, N, groups, softplus;       // groups: of channels, one per workgroup
    int32_t tiles;
    // backward
    const void* dy;
    void *du, *ddelta, *dz, *dB, *dC;
    float *dA, *dD, *dbias;
    int64_t dy_stride, du_stride, dd_stride, dz_stride, db_stride, dc_stride;
    float* backs;                         // workspace [tiles, N, D]: what a tile hands to the gradient of the state it begins with
    float* part_bc;                       // workspace [channel groups, T, 2 N]
    float* part_a;                        // workspace [tiles, N + 2, D]: dA, dD and dbias of a tile
};

constexpr int K = 8;                      // tokens of a block: they are loaded, and their step sizes formed, together

// What a wave's lanes have written to LDS, its lanes read (the LDS unit takes a wave's accesses in order; this holds the compiler
// to it).
__device__ __forceinline__ void lds_in_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// The two channels of a lane: neighbours (one load of two values) where D is even, else 64 apart.
template <bool NEIGHBOURS> struct Channels {
    int d[2];
    bool on[2];
    __device__ __forceinline__ Channels(int group, int lane, int D)
    {
        const int base = group * 128;
        d[0] = base + (NEIGHBOURS ? 2 * lane : lane);
        d[1] = base + (NEIGHBOURS ? 2 * lane + 1 : lane + 64);
        on[0] = d[0] < D;
        on[1] = d[1] < D;
        // lanes and halves without a channel work on a valid one and store nothing
        if (!on[0]) d[0] = NEIGHBOURS ? D - 2 : D - 1;
        if (!on[1]) d[1] = D - 1;
    }
};

template <typename T> struct Two {
    T v[2];
};
template <typename T, bool NEIGHBOURS> __device__ __forceinline__ Two<T> load_two(const T* row, const int (&d)[2])
{
    Two<T> r;
    if constexpr (NEIGHBOURS) {
        __builtin_memcpy(&r, row + d[0], sizeof(r));
    } else {
        r.v[0] = row[d[0]];
        r.v[1] = row[d[1]];
    }
    return r;
}
template <typename T, bool NEIGHBOURS>
__device__ __forceinline__ void store_two(T* row, const Channels<NEIGHBOURS>& c, float a, float b)
{
    if constexpr (NEIGHBOURS) {
        Two<T> r;
        Io<T>::st(&r.v[0], a);
        Io<T>::st(&r.v[1], b);
        if (c.on[0]) __builtin_memcpy(row + c.d[0], &r, sizeof(r));
    } else {
        if (c.on[0]) Io<T>::st(row + c.d[0], a);
        if (c.on[1]) Io<T>::st(row + c.d[1], b);
    }
}

// A wave's 16 states of two channels and A log2(e) for them; states at and behind N are kept at 0 (A = B = C = 0 there).
struct States {
    float h[kStates][2], a2[kStates][2];
};

// States n0 .. n0 + 15 of a row of N in memory; 0 at and behind N.
__device__ __forceinline__ void load_row(float (&out)[kStates], const float* row, int n0, int N)
{
#pragma unroll
    for (int n = 0; n < kStates; ++n) out[n] = 0.f;
    if (N % 4 == 0) {                     // whole groups of four: one load each, at any alignment
#pragma unroll
        for (int n = 0; n < kStates; n += 4)
            if (n0 + n < N) __builtin_memcpy(&out[n], row + n, 16);
    } else {
#pragma unroll
        for (int n = 0; n < kStates; ++n)
            if (n0 + n < N) out[n] = row[n];
    }
}

__device__ __forceinline__ void load_a(States& s, const float* A, const int (&d)[2], int n0, int N)
{
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        float row[kStates];
        load_row(row, A + (int64_t)d[c] * N + n0, n0, N);
#pragma unroll
        for (int n = 0; n < kStates; ++n) s.a2[n][c] = row[n] * kLog2e;
    }
}

// Tokens of a block, as stored.
template <typename T> struct Block {
    Two<T> u[K], delta[K], z[K], dy[K];
    float b[kStates * K / 64], c[kStates * K / 64];    // this lane's part of B and C
};

// B and C of a block go to LDS as binary32 [state][token]: a lane brings one token's states lane / 8, + 8 (16 states, 8 tokens).
// (what a kernel does not ask for it leaves out)
template <typename T, bool WITH_C, bool GATED, bool BACKWARD, bool NEIGHBOURS>
__device__ __forceinline__ void request(Block<T>& k, const PackedScanArgs& a, const Channels<NEIGHBOURS>& c, int n0, int first, int count)
{
#pragma unroll
    for (int t = 0; t < K; ++t) {
        const int64_t row = first + min(t, count - 1);       // rows behind the piece are replaced by its last
        k.u[t] = load_two<T, NEIGHBOURS>(static_cast<const T*>(a.u) + row * a.u_stride, c.d);
        k.delta[t] = load_two<T, NEIGHBOURS>(static_cast<const T*>(a.delta) + row * a.d_stride, c.d);
        if constexpr (BACKWARD) k.dy[t] = load_two<T, NEIGHBOURS>(static_cast<const T*>(a.dy) + row * a.dy_stride, c.d);
        if constexpr (WITH_C && GATED) k.z[t] = load_two<T, NEIGHBOURS>(static_cast<const T*>(a.z) + row * a.z_stride, c.d);
    }
    const int lane = (int)threadIdx.x & 63, t = lane & (K - 1);
    const int64_t row = first + min(t, count - 1);
#pragma unroll
    for (int i = 0; i < kStates * K / 64; ++i) {
        const int n = n0 + (lane >> 3) + 8 * i;
        const bool on = n < a.N;
        k.b[i] = on ? Io<T>::ld(static_cast<const T*>(a.Bm) + row * a.b_stride + n) : 0.f;
        if constexpr (WITH_C) k.c[i] = on ? Io<T>::ld(static_cast<const T*>(a.Cm) + row * a.c_stride + n) : 0.f;
    }
}

template <typename T, bool WITH_C> __device__ __forceinline__ void stage(const Block<T>& k, float* sb, float* sc)
{
    const int lane = (int)threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < kStates * K / 64; ++i) {
        const int at = ((lane >> 3) + 8 * i) * K + (lane & (K - 1));
        sb[at] = k.b[i];
        if constexpr (WITH_C) sc[at] = k.c[i];
    }
}

// A state's values of B or C for a block, from LDS: the loop over the states reads them one state ahead of their use and lets the
// compiler move nothing from one state to another (it would read all of them first and run out of registers).
template <int C> struct Words {
    float v[C];
};
template <int C> __device__ __forceinline__ Words<C> words(const float* p)
{
    Words<C> w;
#pragma unroll
    for (int i = 0; i < C; i += 4) {
        const float4v q = *reinterpret_cast<const float4v*>(p + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) w.v[i + j] = q[j];
    }
    return w;
}

// Step sizes and their products with u; tokens behind the piece get 0 for both: the state stays as it is.
template <typename T>
__device__ __forceinline__ void steps(const Block<T>& k, const float (&bias)[2], bool sp, int count, float (&dl)[2 * K], float (&dx)[2 * K],
                                      float (&u)[2 * K])
{
#pragma unroll
    for (int t = 0; t < K; ++t)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            u[2 * t + c] = Io<T>::ld(&k.u[t].v[c]);
            dl[2 * t + c] = Io<T>::ld(&k.delta[t].v[c]) + bias[c];
        }
    if (sp) corey_scan::softplus_all<2 * K>(dl);
#pragma unroll
    for (int i = 0; i < 2 * K; ++i) {
        dl[i] = i / 2 < count ? dl[i] : 0.f;
        dx[i] = i / 2 < count ? dl[i] * u[i] : 0.f;          // (a NaN among the replaced rows stays out)
    }
}

// f(GROUPS): the waves of a workgroup, 16 states each.
template <typename F> void by_groups(int64_t N, F&& f)
{
    if (N <= 16) f(std::integral_constant<int, 1>());
    else if (N <= 32) f(std::integral_constant<int, 2>());
    else if (N <= 64) f(std::integral_constant<int, 4>());
    else f(std::integral_constant<int, 8>());
    static_assert(COREY_PACK_MAX_STATE == 8 * kStates, "the widest workgroup holds all states");
}

}  // namespace corey_packed
#endif
