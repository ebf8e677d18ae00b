// corey_scan_packed and corey_scan_packed_step: the selective scan on packed batches [T, D], states by slot.
//
//     dl = softplus(delta + bias);  h[n] <- exp(dl A[n]) h[n] + dl B[n] u;  y = (sum_n C[n] h[n] + D u) silu(z)
//
// Channels lie side by side in memory, so a lane is a channel and walks the tokens one after another: B and C of a token are the same
// for the whole wave and sit in scalar registers, the states stay in vector registers, and nothing is exchanged between lanes.  Per
// token, channel and state that is one exponential and four plain instructions; a SIMD issues the first in 8.4 cycles, the others in 2.3
// where two waves' pair, 4.3 where they do not, so vector issue is the bound (memory moves 8 bytes per token and channel in 16-bit
// storage).
//
// Long sequences are cut into tiles that are walked side by side:
//   k_packed_ends    every tile but a sequence's last, from a zero state: its end state E and the sum of its step sizes
//   k_packed_chain   per sequence, over its tiles: h_k+1 = exp(A sum) h_k + E_k; leaves in E's place the state the tile begins with
//   k_packed_scan    every tile from that state; the last one leaves the sequence's state in its slot
// Sequences of one tile need the last kernel alone: its wave reads the slot before it writes it.  In longer ones k_packed_chain has
// read the slot before any tile writes it.
//
// One sequence of 16384 tokens of 5120 bf16 channels with 16 states and a gate, us: 278 for k_packed_scan, of which the states' work takes
// 176 at the 148 cycles that a state and 8 tokens of a wave take in a loop by themselves (corey_packed_scan.h), the rest is step sizes,
// gates, loads and stores and what waits; 204 for k_packed_ends, 13 for k_packed_chain, 5 for the relay of B and C.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "corey_packed_scan.h"

namespace {

using namespace corey_packed;
using corey_scan::float4v;

constexpr int K = kHalf;                  // tokens of a step of the loop: loaded, and their step sizes formed, together

// WHOLE: every wave has 16 states (N = 16 GROUPS): no state's work stands behind a condition.
template <typename T, int GROUPS, bool WHOLE>
__global__ __launch_bounds__(64 * Shape<GROUPS>::waves, 2) void k_packed_ends(PackedScanArgs a)
{
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
    const int n0 = GROUPS > 1 ? wave * kStates : 0;
    const int tile = (int)(blockIdx.x / (unsigned)a.groups);
    const Piece p = a.ix.tiles[tile];
    if (!a.ix.good() || p.seq < 0 || (p.bits & 2) || n0 >= a.N) return;
    const int d = (int)(blockIdx.x % (unsigned)a.groups) * Shape<GROUPS>::channels + (GROUPS > 1 ? 0 : wave * 64) + lane;
    if (d >= a.D) return;
    const uint32_t off = (uint32_t)d * (uint32_t)sizeof(T);
    Rows<T> u_rows(a.u, a.u_stride, p.first), d_rows(a.delta, a.d_stride, p.first);
    Tokens<T, K> u = load_tokens<T, K>(u_rows, p.count, off), delta = load_tokens<T, K>(d_rows, p.count, off);
    float h[kStates], a2[kStates], sum = 0.f;
    load_row<kStates>(a2, a.A + (int64_t)d * a.N + n0, n0, a.N);
#pragma unroll
    for (int n = 0; n < kStates; ++n) {
        a2[n] = rate(a2[n]);
        h[n] = 0.f;
    }
    const float bias = a.bias ? a.bias[d] : 0.f;
    const float* from = a.bc + (first_block(a.ix, p) * 2 * a.N + n0) * 2 * kHalf;
    for (int t0 = 0; t0 < p.count; t0 += K) {                    // (a tile that is not its sequence's last is whole)
        StatePairs s(from);
        float dl[K], dx[K];
        steps<T, K>(u, delta, bias, a.softplus != 0, K, dl, dx);
        const int left = p.count - t0 - K, on = left > 0 ? K : 0;  // (behind the last block: the same rows again, for nothing)
        u_rows.advance(on);
        d_rows.advance(on);
        u = load_tokens<T, K>(u_rows, K, off);
        delta = load_tokens<T, K>(d_rows, K, off);
#pragma unroll
        for (int t = 0; t < K; ++t) sum += dl[t];
#pragma unroll
        for (int n = 0; n < kStates; ++n) {
            if (!WHOLE && n0 + n >= a.N) continue;
            s.ahead(n);
            float e[K], x[K];
            arguments<K>(dl, a2[n], dx, [&](int t) { return s.at(n).b(t); }, e, x);
#pragma unroll
            for (int t = 0; t < K; ++t) h[n] = fmaf(e[t], h[n], x[t]);
            __builtin_amdgcn_sched_barrier(0);
        }
        from += a.N * 2 * kHalf;
    }
    float* out = a.ends + ((int64_t)tile * a.N + n0) * a.D + d;
#pragma unroll
    for (int n = 0; n < kStates; ++n)
        if (n0 + n < a.N) out[(int64_t)n * a.D] = h[n];
    if (n0 == 0) a.sums[(int64_t)tile * a.D + d] = sum;
}

// A lane is one channel and state of one sequence.  The tiles' values are requested kAhead at a time (48 sequences of up to 64 tiles, 2048
// channels, us: 8 19, 16 21, 32 27).
constexpr int kAhead = 8;
__global__ __launch_bounds__(256) void k_packed_chain(PackedScanArgs a, int columns)
{
    const int which = (int)(blockIdx.x / (unsigned)columns);
    const int64_t col = (int64_t)(blockIdx.x % (unsigned)columns) * 256 + threadIdx.x;
    if (!a.ix.good() || which >= a.ix.head[7] || col >= (int64_t)a.D * a.N) return;
    const int seq = a.ix.longs[which];
    const int first = a.ix.tile_begin[seq], stop = a.ix.tile_begin[seq + 1];
    const int n = (int)(col / a.D), d = (int)(col % a.D);
    const float a2 = rate(a.A[(int64_t)d * a.N + n]);
    const int64_t slot = slot_of(a.slots, seq, a.n_slots), wide = (int64_t)a.N * a.D;
    float h = slot >= 0 ? a.state[(slot * a.D + d) * a.N + n] : 0.f;
    float* e = a.ends + col;
    const float* sums = a.sums + d;
    for (int k0 = first; k0 < stop; k0 += kAhead) {
        float end[kAhead], sum[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t k = min(k0 + i, stop - 2);             // (the last tile has no end state)
            end[i] = e[k * wide];
            sum[i] = sums[k * a.D];
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (k0 + i < stop) {
                e[(k0 + i) * wide] = h;
                h = h == 0.f ? end[i] : fmaf(fast_exp2(a2 * sum[i]), h, end[i]);   // (a decay may have overflowed, step sizes below 0)
            }
        }
    }
}

template <typename T, bool GATED, int GROUPS, bool WHOLE>
__global__ __launch_bounds__(64 * Shape<GROUPS>::waves, 2) void k_packed_scan(PackedScanArgs a)
{
    __shared__ float s_part[GROUPS > 1 ? GROUPS - 1 : 1][GROUPS > 1 ? K * 64 : 1];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
    const int n0 = GROUPS > 1 ? wave * kStates : 0;
    const int tile = (int)(blockIdx.x / (unsigned)a.groups);
    const Piece p = a.ix.tiles[tile];
    if (!a.ix.good() || p.seq < 0) return;                       // (the same for every wave of the workgroup)
    const int d = (int)(blockIdx.x % (unsigned)a.groups) * Shape<GROUPS>::channels + (GROUPS > 1 ? 0 : wave * 64) + lane;
    if (d >= a.D) return;
    const bool states = n0 < a.N;                                // (a workgroup's last waves may have no states)
    const uint32_t off = (uint32_t)d * (uint32_t)sizeof(T);
    Rows<T> u_rows(a.u, a.u_stride, p.first), d_rows(a.delta, a.d_stride, p.first), z_rows(GATED ? a.z : a.u, GATED ? a.z_stride : 0, p.first),
        y_rows(a.y, a.y_stride, p.first);
    Tokens<T, K> u = load_tokens<T, K>(u_rows, p.count, off), delta = load_tokens<T, K>(d_rows, p.count, off);
    float h[kStates], a2[kStates];
    load_row<kStates>(a2, a.A + (int64_t)d * a.N + n0, n0, a.N);
#pragma unroll
    for (int n = 0; n < kStates; ++n) a2[n] = rate(a2[n]);
    const float bias = a.bias ? a.bias[d] : 0.f, skip = a.Dv && n0 == 0 ? a.Dv[d] : 0.f;
    // the state the tile begins with
    if (p.bits == 3) {
        const int64_t slot = slot_of(a.slots, p.seq, a.n_slots);
        if (slot >= 0) load_row<kStates>(h, a.state + (slot * a.D + d) * a.N + n0, n0, a.N);
        else {
#pragma unroll
            for (int n = 0; n < kStates; ++n) h[n] = 0.f;
        }
    } else {
        const float* start = a.ends + ((int64_t)tile * a.N + n0) * a.D + d;
#pragma unroll
        for (int n = 0; n < kStates; ++n) h[n] = n0 + n < a.N ? start[(int64_t)n * a.D] : 0.f;
    }
    const float* from = a.bc + (first_block(a.ix, p) * 2 * a.N + (states ? n0 : 0)) * 2 * kHalf;
    for (int t0 = 0; t0 < p.count; t0 += K) {
        const int count = p.count - t0;
        StatePairs s(from);
        float dl[K], dx[K], acc[K];
        Tokens<T, K> z;                                          // (needed at the end: requested now, not with the block before)
        if constexpr (GATED) {
            z = load_tokens<T, K>(z_rows, count, off);
            z_rows.advance(K);
        }
        steps<T, K>(u, delta, bias, a.softplus != 0, count, dl, dx);
#pragma unroll
        for (int t = 0; t < K; ++t) acc[t] = skip * u.at(t);     // the skip term D u opens the sum over the states
        const bool more = count > K;                             // (behind the last block: the same rows again, for nothing)
        u_rows.advance(more ? K : 0);
        d_rows.advance(more ? K : 0);
        u = load_tokens<T, K>(u_rows, more ? count - K : count, off);
        delta = load_tokens<T, K>(d_rows, more ? count - K : count, off);
#pragma unroll
        for (int n = 0; n < kStates; ++n) {
            if (!WHOLE && n0 + n >= a.N) continue;
            s.ahead(n);
            float e[K], x[K];
            arguments<K>(dl, a2[n], dx, [&](int t) { return s.at(n).b(t); }, e, x);
#pragma unroll
            for (int t = 0; t < K; ++t) {
                h[n] = fmaf(e[t], h[n], x[t]);
                acc[t] = fmaf(s.at(n).c(t), h[n], acc[t]);
                // a state's share of the sums is added here: left to itself the compiler moves a token's sum over the states into the
                // branch that stores it, and keeps the states of all tokens until then
                asm volatile("" : "+v"(acc[t]), "+v"(h[n]));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        from += a.N * 2 * kHalf;
        if constexpr (GROUPS > 1) {                              // the sum over the waves' states; wave 0 finishes
            __syncthreads();
            if (wave != 0) {
#pragma unroll
                for (int t = 0; t < K; ++t) s_part[wave - 1][t * 64 + lane] = acc[t];
            }
            __syncthreads();
            if (wave != 0) continue;
            for (int w = 0; w + 1 < GROUPS; ++w) {
#pragma unroll
                for (int t = 0; t < K; ++t) acc[t] += s_part[w][t * 64 + lane];
            }
        }
        if constexpr (GATED) {
            float g[K];
            gates<T, K>(z, g);
#pragma unroll
            for (int t = 0; t < K; ++t) acc[t] *= g[t];
        }
        store_tokens<T, K>(y_rows, count, off, acc);
        y_rows.advance(K);
    }
    if (!(p.bits & 2)) return;
    const int64_t to = slot_of(a.slots_out, p.seq, a.n_slots);
    if (to < 0) return;
    float* out = a.state + (to * a.D + d) * a.N + n0;
    if (a.N % 4 == 0) {
#pragma unroll
        for (int n = 0; n < kStates; n += 4) {
            const float q[4] = {h[n], h[n + 1], h[n + 2], h[n + 3]};
            if (n0 + n < a.N) __builtin_memcpy(out + n, q, sizeof(q));
        }
    } else {
#pragma unroll
        for (int n = 0; n < kStates; ++n)
            if (n0 + n < a.N) out[n] = h[n];
    }
}

// One token of every sequence.  As the state's update of a whole batch: a row of N states is spread over 2^k lanes of four states.
struct StepArgs {
    float* state;
    const int32_t *slots, *slots_out;
    const void *x, *delta, *Bt, *Ct, *z;
    const float *A, *Dv, *bias;
    void* y;
    int64_t x_stride, d_stride, b_stride, c_stride, z_stride, y_stride, n_slots;
    uint32_t rows, D;
    int32_t N, lpr_log2, softplus;
};

// States in whole groups of four in aligned memory: U sets of 256 lanes a workgroup, every load of theirs issued before any use.  Bound by
// memory (8 bytes a state).  One set, two and four, states from HBM, us, sequences of 5120 bf16 channels with 16 states: 16 (1280 sets)
// 6.5, 6.7, 10; 40 12.2, 10.5, 13.7; 64 17.3, 14.6, 22; 512 115, 100, 132 (3.6 TB/s; a copy reaches 4.9); of 1536 channels 40 (960 sets) 5.6,
// 5.7; 64 (1536) 7.0, 6.6; binary32, 5120: 16 6.3, 5.9; 64 17.3, 14.0; 512 110, 97.  The line between one and two is that of 16-bit rows
// (in binary32 two win by 0.4 us at 1280 sets already).
constexpr uint64_t kManySets = 1400;
template <typename T, int U>
__global__ __launch_bounds__(256) void k_packed_step(StepArgs a)
{
    const int LPR = 1 << a.lpr_log2, j = (int)threadIdx.x & (LPR - 1);
    const bool on = 4 * j < a.N;
    const int n = on ? 4 * j : 0;                                // lanes without a group load the row's first and store nothing
    bool active[U];
    uint32_t b[U], d[U];
    int64_t from[U], to[U];
    float4v h[U], av[U];
    T bv[U][4], cv[U][4], xr[U], dr[U], zr[U];
    float bias[U], skip[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const uint32_t r = (uint32_t)((((uint64_t)blockIdx.x * U + k) * 256 + threadIdx.x) >> a.lpr_log2);
        active[k] = r < a.rows;                                  // whole rows are active or not: LPR divides the wave
        const uint32_t row = active[k] ? r : a.rows - 1;
        b[k] = row / a.D;
        d[k] = row - b[k] * a.D;
        from[k] = slot_of(a.slots, (int)b[k], a.n_slots);
        to[k] = slot_of(a.slots_out, (int)b[k], a.n_slots);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
        h[k] = *reinterpret_cast<const float4v*>(a.state + ((from[k] >= 0 ? from[k] : 0) * a.D + d[k]) * a.N + n);
        __builtin_memcpy(&av[k], a.A + (int64_t)d[k] * a.N + n, sizeof(av[k]));
        __builtin_memcpy(bv[k], static_cast<const T*>(a.Bt) + (int64_t)b[k] * a.b_stride + n, sizeof(bv[k]));
        __builtin_memcpy(cv[k], static_cast<const T*>(a.Ct) + (int64_t)b[k] * a.c_stride + n, sizeof(cv[k]));
        xr[k] = static_cast<const T*>(a.x)[(int64_t)b[k] * a.x_stride + d[k]];
        dr[k] = static_cast<const T*>(a.delta)[(int64_t)b[k] * a.d_stride + d[k]];
        zr[k] = a.z ? static_cast<const T*>(a.z)[(int64_t)b[k] * a.z_stride + d[k]] : T(0);
        bias[k] = a.bias ? a.bias[d[k]] : 0.f;
        skip[k] = a.Dv ? a.Dv[d[k]] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const float xv = Io<T>::ld(&xr[k]);
        float dl = Io<T>::ld(&dr[k]) + bias[k];
        if (a.softplus) dl = softplus(dl);
        const float dx = dl * xv;
        float acc = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float h0 = from[k] >= 0 ? h[k][i] : 0.f;
            h[k][i] = fmaf(fast_exp2(dl * (av[k][i] * kLog2e)), h0, dx * Io<T>::ld(&bv[k][i]));
            acc = fmaf(Io<T>::ld(&cv[k][i]), h[k][i], acc);
        }
        if (!on) acc = 0.f;
        if (active[k] && on && to[k] >= 0) *reinterpret_cast<float4v*>(a.state + (to[k] * a.D + d[k]) * a.N + n) = h[k];
        for (int m = LPR >> 1; m >= 1; m >>= 1) acc += __shfl_xor(acc, m);
        if (active[k] && j == 0) {
            float yv = a.Dv ? fmaf(skip[k], xv, acc) : acc;
            if (a.z) yv *= silu(Io<T>::ld(&zr[k]));
            Io<T>::st(static_cast<T*>(a.y) + (int64_t)b[k] * a.y_stride + d[k], yv);
        }
    }
}

// Any N and any alignment of the states: value by value.
template <typename T>
__global__ __launch_bounds__(256) void k_packed_step_any(StepArgs a)
{
    const uint64_t gid = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const int LPR = 1 << a.lpr_log2, j = (int)(gid & (uint64_t)(LPR - 1)), n = 4 * j;
    const uint32_t r = (uint32_t)(gid >> a.lpr_log2);
    const bool active = r < a.rows;                              // whole rows are active or not: LPR divides the wave
    float acc = 0.f, xv = 0.f;
    uint32_t b = 0, d = 0;
    if (active) {
        b = r / a.D;
        d = r - b * a.D;
        const int64_t from = slot_of(a.slots, (int)b, a.n_slots), to = slot_of(a.slots_out, (int)b, a.n_slots);
        xv = Io<T>::ld(static_cast<const T*>(a.x) + (int64_t)b * a.x_stride + d);
        float dl = Io<T>::ld(static_cast<const T*>(a.delta) + (int64_t)b * a.d_stride + d) + (a.bias ? a.bias[d] : 0.f);
        if (a.softplus) dl = softplus(dl);
        const float dx = dl * xv;
        for (int i = n; i < a.N && i < n + 4; ++i) {
            const float h0 = from >= 0 ? a.state[(from * a.D + d) * a.N + i] : 0.f;
            const float bi = Io<T>::ld(static_cast<const T*>(a.Bt) + (int64_t)b * a.b_stride + i);
            const float hn = fmaf(fast_exp2(dl * (a.A[(int64_t)d * a.N + i] * kLog2e)), h0, dx * bi);
            if (to >= 0) a.state[(to * a.D + d) * a.N + i] = hn;
            acc = fmaf(Io<T>::ld(static_cast<const T*>(a.Ct) + (int64_t)b * a.c_stride + i), hn, acc);
        }
    }
    for (int m = LPR >> 1; m >= 1; m >>= 1) acc += __shfl_xor(acc, m);
    if (active && j == 0) {
        float yv = a.Dv ? fmaf(a.Dv[d], xv, acc) : acc;
        if (a.z) yv *= silu(Io<T>::ld(static_cast<const T*>(a.z) + (int64_t)b * a.z_stride + d));
        Io<T>::st(static_cast<T*>(a.y) + (int64_t)b * a.y_stride + d, yv);
    }
}

}  // namespace

// Tiles are what runs side by side.  A tile costs its tokens and some more for the state it begins with; a SIMD with m waves takes m
// times that, and more than its share with fewer than four (nothing issues beside them); and a sequence's tiles are chained one after
// another.  Of the tiles of whole blocks the one with the least of it, counting half a tile a sequence for the ends that fill none.  One
// sequence of 16384 tokens, 5120 channels: 320 (four waves a SIMD); tiles of 64, 128, 192, 256, 288, 320, 384, 512, 1024 tokens take 467,
// 440, 451, 456, 499, 456, 529, 545, 777 us.
// Where half a tile a sequence fills the GPU a tile takes whole sequences, up to four times their mean length: cut, they are walked
// twice (160 sequences of 5120 channels, lengths of 100 spread over a factor of 20, us: 466 in tiles of 272, 328 in one tile each), but one
// that is much longer than the rest is walked by too few waves if it is not (16384 tokens and 200 sequences of one: 1024 915, 336 some
// 520, 160 474; 800 and 200 of one: 1024 299, 32 89).  It loses where the longest lies between that and 1024 (exponential lengths of
// 100: 432 518, 1024 397; spread over a factor of 100: 400 595, 1024 419) and two launches that find nothing to begin (200 sequences of
// three tokens: 1024 51, 32 58).
extern "C" int32_t corey_pack_tile(int64_t S, int64_t T, int64_t D, int64_t N, int backward)
{
    if (S < 1 || T < 1 || T > INT32_MAX || D < 1 || D > COREY_PACK_MAX_CHANNELS || N < 1 || N > COREY_PACK_MAX_STATE) return 0;
    constexpr double kSimds = 4. * 256.;
    const double waves = (double)((D + 63) / 64) * (double)((N + 15) / 16), length = (double)T / (double)S;
    // backward: 8192 tokens of 2048 bf16 channels in 11 sequences, tiles of 16, 32, 48, 64 tokens 477, 375, 338, 370 us; 2048 of 1536 in
    // four 112, 99, 124, 130; 16384 of 4096 in four 1682, 1312, 1199, 1167; 16384 of 64 in one 233, 157, 158, 156
    const double more = backward ? 8. : 6., chained = backward ? 0.15 : 0.6, slack = backward ? 0. : 0.1;
    const auto cost = [&](double tile) {
        const double m = std::max(1., std::ceil((T / tile + 0.5 * S) * waves / kSimds - slack));
        return (m == 1. ? 1.75 : m == 2. ? 2.3 : m) * (tile + more) + chained * length / tile;
    };
    const int32_t most = !backward ? 1024 : N > 64 ? 32 : 64;
    if (!backward && 0.5 * S * waves >= 4.5 * kSimds)
        return (int32_t)std::min<double>(most, std::max(2., std::ceil(4. * length / COREY_PACK_BLOCK)) * COREY_PACK_BLOCK);
    int32_t best = COREY_PACK_BLOCK;
    for (int32_t tile = 2 * COREY_PACK_BLOCK; tile <= most; tile += COREY_PACK_BLOCK)
        if (cost(tile) < cost(best)) best = tile;
    return best;
}

namespace {
// The workspace's parts, in floats.
struct Space {
    int64_t bc, ends, sums, all;
};
Space space(const Layout& l, int64_t T, int32_t tile, int64_t D, int64_t N)
{
    const int64_t tiles = T > tile ? l.max_tiles : 0;            // (carried only where a sequence can have a second tile)
    Space s;
    s.bc = 0;
    s.ends = s.bc + l.max_blocks * N * 32 + 48;                  // (the loop over the states asks for three more than there are)
    s.sums = s.ends + tiles * N * D;
    s.all = s.sums + tiles * D;
    return s;
}
}  // namespace

extern "C" size_t corey_scan_packed_workspace(const corey_pack* pack, int64_t D, int64_t N)
{
    Index ix;
    if (D < 1 || D > COREY_PACK_MAX_CHANNELS || N < 1 || N > COREY_PACK_MAX_STATE || index_of("corey_scan_packed_workspace", pack, &ix)) return 0;
    return (size_t)space(layout(pack->S, pack->T, pack->tile), pack->T, pack->tile, D, N).all * 4;
}

extern "C" int corey_scan_packed(const void* u, int64_t u_stride, const void* delta, int64_t delta_stride, const float* A, const void* Bm,
                                 int64_t B_stride, const void* Cm, int64_t C_stride, const float* Dv, const void* z, int64_t z_stride,
                                 const float* delta_bias, int delta_softplus, float* state, int64_t n_slots, const int32_t* slots,
                                 const int32_t* slots_out, const corey_pack* pack, void* y, int64_t y_stride, corey_dtype dt, int64_t D,
                                 int64_t N, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    using corey::fail;
    const char* who = "corey_scan_packed";
    if (!u || !delta || !A || !Bm || !Cm || !y) return fail(COREY_ENULL, "%s: u, delta, A, Bm, Cm and y are required", who);
    if (!good_dtype(dt)) return fail(COREY_EINVAL, "%s: unknown dtype %d", who, (int)dt);
    if (D < 1 || D > COREY_PACK_MAX_CHANNELS || N < 1) return fail(COREY_ESHAPE, "%s: 1 <= D <= %d and N >= 1 required", who, COREY_PACK_MAX_CHANNELS);
    if (N > COREY_PACK_MAX_STATE) return fail(COREY_EUNSUPPORTED, "%s: N above %d", who, COREY_PACK_MAX_STATE);
    if (!good_stride(u_stride, D) || !good_stride(delta_stride, D) || !good_stride(y_stride, D) || (z && !good_stride(z_stride, D)) ||
        !good_stride(B_stride, N) || !good_stride(C_stride, N))
        return fail(COREY_ESHAPE, "%s: rows must be at least D (B and C: N) apart", who);
    if ((slots || slots_out) && (!state || n_slots < 1)) return fail(COREY_ENULL, "%s: slots need a pool of states", who);
    if (y == u || y == delta || y == Bm || y == Cm || y == z) return fail(COREY_EINVAL, "%s: y may not be an input", who);
    PackedScanArgs a = {};
    if (int e = index_of(who, pack, &a.ix)) return e;
    if (!workspace || workspace_bytes < corey_scan_packed_workspace(pack, D, N) || reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
        return fail(COREY_EWORKSPACE, "%s: workspace missing, misaligned or smaller than corey_scan_packed_workspace()", who);
    const Layout l = layout(pack->S, pack->T, pack->tile);
    a.u = u; a.delta = delta; a.Bm = Bm; a.Cm = Cm; a.z = z;
    a.A = A; a.Dv = Dv; a.bias = delta_bias;
    a.y = y;
    a.state = state; a.slots = slots; a.slots_out = slots_out ? slots_out : slots; a.n_slots = n_slots;
    a.u_stride = u_stride; a.d_stride = delta_stride; a.b_stride = B_stride; a.c_stride = C_stride; a.z_stride = z_stride; a.y_stride = y_stride;
    const Space w = space(l, pack->T, pack->tile, D, N);
    a.bc = static_cast<float*>(workspace) + w.bc;
    a.ends = static_cast<float*>(workspace) + w.ends;
    a.sums = static_cast<float*>(workspace) + w.sums;
    a.D = (int32_t)D; a.N = (int32_t)N;
    a.softplus = delta_softplus ? 1 : 0;
    a.blocks = (int32_t)l.max_blocks;
    a.groups = (int32_t)channel_groups(D, N);
    const int64_t grid = l.max_tiles * a.groups, columns = (D * N + 255) / 256, relay = (l.max_blocks * N * 32 + 255) / 256;
    if (!good_grid(grid, 64 * waves_of(N)) || !good_grid(relay, 256) || !good_grid(columns * l.max_longs, 256)) return fail(COREY_ESHAPE, "%s: T * D is too large", who);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    by_type(dt, [&](auto t) {
        using T = decltype(t);
        k_packed_relay<T><<<(unsigned)relay, 256, 0, stream>>>(a);
        by_groups(N, [&](auto g) {
            constexpr int G = decltype(g)::value;
            const auto go = [&](auto whole) {
                constexpr bool W = decltype(whole)::value;
                if (pack->T > pack->tile) {
                    k_packed_ends<T, G, W><<<(unsigned)grid, 64 * Shape<G>::waves, 0, stream>>>(a);
                    k_packed_chain<<<(unsigned)(columns * l.max_longs), 256, 0, stream>>>(a, (int)columns);
                }
                if (z) k_packed_scan<T, true, G, W><<<(unsigned)grid, 64 * Shape<G>::waves, 0, stream>>>(a);
                else k_packed_scan<T, false, G, W><<<(unsigned)grid, 64 * Shape<G>::waves, 0, stream>>>(a);
            };
            if (N == G * kStates) go(std::true_type());
            else go(std::false_type());
        });
    });
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? corey::hip_fail(e, "corey_scan_packed launch") : COREY_OK;
}

extern "C" int corey_scan_packed_step(float* state, int64_t n_slots, const int32_t* slots, const int32_t* slots_out, const void* x,
                                      int64_t x_stride, const void* delta, int64_t delta_stride, const float* A, const void* Bt,
                                      int64_t B_stride, const void* Ct, int64_t C_stride, const float* Dv, const void* z, int64_t z_stride,
                                      const float* delta_bias, int delta_softplus, void* y, int64_t y_stride, corey_dtype dt, int64_t S,
                                      int64_t D, int64_t N, void* hip_stream)
{
    using corey::fail;
    const char* who = "corey_scan_packed_step";
    if (!state || !slots || !x || !delta || !A || !Bt || !Ct || !y)
        return fail(COREY_ENULL, "%s: state, slots, x, delta, A, Bt, Ct and y are required", who);
    if (!good_dtype(dt)) return fail(COREY_EINVAL, "%s: unknown dtype %d", who, (int)dt);
    if (S < 1 || D < 1 || N < 1 || n_slots < 1 || N > COREY_MAX_STATE)
        return fail(COREY_ESHAPE, "%s: S, D, n_slots >= 1 and 1 <= N <= %d required", who, COREY_MAX_STATE);
    if ((double)S * (double)D >= 33554432.0) return fail(COREY_ESHAPE, "%s: S*D must stay below 2^25", who);
    if (!good_stride(x_stride, D) || !good_stride(delta_stride, D) || !good_stride(y_stride, D) || (z && !good_stride(z_stride, D)) ||
        !good_stride(B_stride, N) || !good_stride(C_stride, N))
        return fail(COREY_ESHAPE, "%s: rows must be at least D (Bt and Ct: N) apart", who);
    if (reinterpret_cast<uintptr_t>(state) % 4 != 0) return fail(COREY_EINVAL, "%s: state must be 4-byte aligned", who);
    if (y == x || y == delta || y == Bt || y == Ct || y == z) return fail(COREY_EINVAL, "%s: y may not be an input", who);
    StepArgs a;
    a.state = state; a.slots = slots; a.slots_out = slots_out ? slots_out : slots;
    a.x = x; a.delta = delta; a.Bt = Bt; a.Ct = Ct; a.z = z;
    a.A = A; a.Dv = Dv; a.bias = delta_bias;
    a.y = y;
    a.x_stride = x_stride; a.d_stride = delta_stride; a.b_stride = B_stride; a.c_stride = C_stride; a.z_stride = z_stride; a.y_stride = y_stride;
    a.n_slots = n_slots;
    a.rows = (uint32_t)(S * D);
    a.D = (uint32_t)D;
    a.N = (int32_t)N;
    a.lpr_log2 = 0;
    while ((1 << a.lpr_log2) < (N + 3) / 4) ++a.lpr_log2;
    a.softplus = delta_softplus ? 1 : 0;
    const uint64_t sets = (((uint64_t)(S * D) << a.lpr_log2) + 255) / 256;
    const bool vector = N % 4 == 0 && reinterpret_cast<uintptr_t>(state) % 16 == 0;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    by_type(dt, [&](auto t) {
        using T = decltype(t);
        if (!vector) k_packed_step_any<T><<<(unsigned)sets, 256, 0, stream>>>(a);
        else if (sets > kManySets) k_packed_step<T, 2><<<(unsigned)((sets + 1) / 2), 256, 0, stream>>>(a);
        else k_packed_step<T, 1><<<(unsigned)sets, 256, 0, stream>>>(a);
    });
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? corey::hip_fail(e, "corey_scan_packed_step launch") : COREY_OK;
}
