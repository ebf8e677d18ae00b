// corey_scan_packed_bwd: the gradients of the selective scan on packed batches, from dy and the scan's inputs.
//
//     a_t = exp(dl_t A), h_t = a_t h_{t-1} + dl_t B_t u_t, s_t = sum_n C_t h_t + D u_t, y_t = s_t silu(z_t);   ds = dy silu(z)
//     g_t = ds_t C_t + a_{t+1} g_{t+1}                        (the gradient of h_t)
//     dC_t = sum_d ds h,  dB_t = sum_d g dl u,  ddl = sum_n g (u B + A a h_{t-1}),  du = D ds + dl sum_n g B,  dA = sum_t g dl a h_{t-1}
//
// Sequences are cut into tiles of at most 64 tokens that are walked side by side:
//   k_packed_bwd_ends   every tile of more than one block of 16 tokens or of a longer sequence: its end state E from zero, those at
//                       the starts of its blocks, the gradient G that it hands to the state it begins with when none comes from
//                       behind, and the sums of its step sizes
//   k_packed_bwd_chain  per sequence, over its tiles: forward h_k+1 = exp(A sum) h_k + E_k, backward g_k-1 = exp(A sum) g_k + G_k
//   k_packed_bwd        every tile, block by block from the last, state by state: the block begins with exp(A sum) times the tile's first
//                       state and its own from zero; from there the block's decays and states forward, its gradients backward.
//                       Sums over states stay in the lane (a lane is a channel); sums over channels (dB, dC) are folded over the
//                       wave's lanes, over the workgroup's waves in LDS, and written per workgroup
//   k_packed_bwd_bc, k_packed_bwd_a   add up the workgroups' dB and dC, and the tiles' dA, dD and dbias, always in the same order
// Per token, channel and state k_packed_bwd issues some 21 vector instructions, one of them an exponential, and k_packed_bwd_ends 8; vector
// issue is the bound, two waves a SIMD (some 240 registers and 19 KB of LDS a wave).  8192 tokens of 2048 bf16 channels with 16 states in 11
// sequences, us: 241, ends 85, chain 21, dA 8, dB and dC 8, relay 5.  (With the states at block starts formed again in k_packed_bwd 308 and
// ends 74; before its loop took two states a turn 254.  Leaving parts out: the folds take 45, a block's end with its stores 50.)
#include <hip/hip_runtime.h>

#include "corey_packed_scan.h"

namespace {

using namespace corey_packed;
using corey_scan::dpp_move;

constexpr int kTok = kBlock;              // tokens of a block
constexpr int kMaxBackTile = 64;
constexpr int K = kHalf;                  // tokens of a step of k_packed_bwd_ends

template <typename T, bool GATED, int GROUPS, bool WHOLE>
__global__ __launch_bounds__(64 * Shape<GROUPS>::waves, 2) void k_packed_bwd_ends(PackedScanArgs a)
{
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
    const int n0 = GROUPS > 1 ? wave * kStates : 0;
    const int tile = (int)(blockIdx.x / (unsigned)a.groups);
    const Piece p = a.ix.tiles[tile];
    if (!a.ix.good() || p.seq < 0 || (p.bits == 3 && p.count <= kTok) || n0 >= a.N) return;
    const int d = (int)(blockIdx.x % (unsigned)a.groups) * Shape<GROUPS>::channels + (GROUPS > 1 ? 0 : wave * 64) + lane;
    if (d >= a.D) return;
    const uint32_t off = (uint32_t)d * (uint32_t)sizeof(T);
    Rows<T> u_rows(a.u, a.u_stride, p.first), d_rows(a.delta, a.d_stride, p.first), y_rows(a.dy, a.dy_stride, p.first),
        z_rows(GATED ? a.z : a.u, GATED ? a.z_stride : 0, p.first);
    Tokens<T, K> u, delta, dy, z;
    const auto request = [&](int tokens, int count) {
        u_rows.advance(tokens);
        d_rows.advance(tokens);
        y_rows.advance(tokens);
        u = load_tokens<T, K>(u_rows, count, off);
        delta = load_tokens<T, K>(d_rows, count, off);
        dy = load_tokens<T, K>(y_rows, count, off);
        if constexpr (GATED) {
            z_rows.advance(tokens);
            z = load_tokens<T, K>(z_rows, count, off);
        }
    };
    request(0, p.count);
    float h[kStates], a2[kStates], back[kStates], sum = 0.f;
    load_row<kStates>(a2, a.A + (int64_t)d * a.N + n0, n0, a.N);
#pragma unroll
    for (int n = 0; n < kStates; ++n) {
        a2[n] = rate(a2[n]);
        h[n] = back[n] = 0.f;
    }
    const float bias = a.bias ? a.bias[d] : 0.f;
    const float* from = a.bc + (first_block(a.ix, p) * 2 * a.N + n0) * 2 * kHalf;
    const int64_t starts = (int64_t)tile * (a.ix.tile / kTok - 1);
    for (int t0 = 0; t0 < p.count; t0 += K) {
        const int count = p.count - t0;
        if (t0 != 0 && t0 % kTok == 0) {                         // a block but the tile's first begins
            const int64_t at = starts + t0 / kTok - 1;
            float* start = a.starts + (at * a.N + n0) * a.D + d;
#pragma unroll
            for (int n = 0; n < kStates; ++n)
                if (n0 + n < a.N) start[(int64_t)n * a.D] = h[n];
            if (n0 == 0) a.start_sums[at * a.D + d] = sum;
        }
        StatePairs s(from);
        float dl[K], dx[K], ds[K];
        steps<T, K>(u, delta, bias, a.softplus != 0, count, dl, dx);
        if constexpr (GATED) gates<T, K>(z, ds);
#pragma unroll
        for (int t = 0; t < K; ++t) {
            ds[t] = GATED ? ds[t] * dy.at(t) : dy.at(t);
            if (count < K) ds[t] = t < count ? ds[t] : 0.f;
        }
        const float before = sum;                                // the decay up to here is exp(A before)
#pragma unroll
        for (int t = 0; t < K; ++t) sum += dl[t];
        request(count > K ? K : 0, count > K ? count - K : count);       // (behind the last block: the same rows again, for nothing)
#pragma unroll
        for (int n = 0; n < kStates; ++n) {
            if (!WHOLE && n0 + n >= a.N) continue;
            s.ahead(n);
            float e[K], x[K], g = 0.f;
            arguments<K>(dl, a2[n], dx, [&](int t) { return s.at(n).b(t); }, e, x);
#pragma unroll
            for (int t = 0; t < K; ++t) {
                h[n] = fmaf(e[t], h[n], x[t]);
                const int r = K - 1 - t;                         // (and the gradients from the last token back)
                g = fmaf(s.at(n).c(r), ds[r], g) * e[r];
            }
            back[n] = g == 0.f ? back[n] : fmaf(fast_exp2(before * a2[n]), g, back[n]);   // (as in the chain: the decay may have overflowed)
            __builtin_amdgcn_sched_barrier(0);
        }
        from += a.N * 2 * kHalf;
    }
    if (p.bits == 3) return;
    const int64_t at = ((int64_t)tile * a.N + n0) * a.D + d;
#pragma unroll
    for (int n = 0; n < kStates; ++n) {
        if (n0 + n < a.N) {
            a.ends[at + (int64_t)n * a.D] = h[n];
            a.backs[at + (int64_t)n * a.D] = back[n];
        }
    }
    if (n0 == 0) a.sums[(int64_t)tile * a.D + d] = sum;
}

// A lane is one channel and state of one sequence, in one direction.  Leaves the state each tile begins with in `ends`, the gradient
// that comes to its end from behind in `backs`.
constexpr int kAhead = 8;
__global__ __launch_bounds__(256) void k_packed_bwd_chain(PackedScanArgs a, int columns)
{
    const bool forward = (blockIdx.x & 1) == 0;
    const int which = (int)((blockIdx.x >> 1) / (unsigned)columns);
    const int64_t col = (int64_t)((blockIdx.x >> 1) % (unsigned)columns) * 256 + threadIdx.x;
    if (!a.ix.good() || which >= a.ix.head[7] || col >= (int64_t)a.D * a.N) return;
    const int seq = a.ix.longs[which];
    const int first = a.ix.tile_begin[seq], stop = a.ix.tile_begin[seq + 1], tiles = stop - first;
    const int n = (int)(col / a.D), d = (int)(col % a.D);
    const float a2 = rate(a.A[(int64_t)d * a.N + n]);
    const int64_t wide = (int64_t)a.N * a.D;
    float* e = (forward ? a.ends : a.backs) + col;
    const float* sums = a.sums + d;
    float h = 0.f;
    for (int k0 = 0; k0 < tiles; k0 += kAhead) {
        float end[kAhead], sum[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int k = min(k0 + i, tiles - 1);
            const int64_t row = forward ? first + k : stop - 1 - k;
            end[i] = e[row * wide];
            sum[i] = sums[row * a.D];
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (k0 + i < tiles) {
                e[(int64_t)(forward ? first + k0 + i : stop - 1 - k0 - i) * wide] = h;
                h = h == 0.f ? end[i] : fmaf(fast_exp2(a2 * sum[i]), h, end[i]);   // (a decay may have overflowed, step sizes below 0)
            }
        }
    }
}

// Sums of 16 values of every lane over the wave's 64 lanes, by way of LDS: a value's 64 parts are a row there, four lanes add up a
// quarter of it each and then their sums.  (Halving over lanes in registers takes 24 swaps and selects of 8 and 4 cycles a fold where
// this takes 15 additions and 2 DPP additions; and an eighth of the LDS unit's time.)  The row's length keeps the reads of 16 bytes from
// meeting in the same banks.  The LDS unit takes a wave's accesses in order, so nothing waits between a lane's write and another's
// read; the compiler is held to the order.
constexpr int kFoldRow = 68, kFoldRows = kTok * kFoldRow;
__device__ __forceinline__ void lds_in_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}
__device__ __forceinline__ void fold_put(float* buf, const float (&v)[kTok], int lane)
{
    lds_in_order();
#pragma unroll
    for (int t = 0; t < kTok; ++t) buf[t * kFoldRow + lane] = v[t];
    lds_in_order();
}
struct Quarter {                          // of the row of value lane / 4
    corey_scan::float4v v[4];
};
__device__ __forceinline__ Quarter fold_read(const float* buf, int lane)
{
    const corey_scan::float4v* row = reinterpret_cast<const corey_scan::float4v*>(buf + (lane >> 2) * kFoldRow + (lane & 3) * 16);
    Quarter q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q.v[i] = row[i];
    return q;
}
// every lane leaves with the sum of value lane / 4
__device__ __forceinline__ float fold_sum(const Quarter& q)
{
    const corey_scan::float4v a = q.v[0] + q.v[1], b = q.v[2] + q.v[3], c = a + b;
    float r = (c[0] + c[1]) + (c[2] + c[3]);
    constexpr int kXor2 = 0x4e, kXor1 = 0xb1;                    // quad_perm
    r += dpp_move<kXor2>(r);
    r += dpp_move<kXor1>(r);
    return r;
}

// The loop over the states is a loop (unrolled it is 50 KB of instructions, more than the instruction cache feeds), so what belongs to
// a state from block to block stays out of registers: its gradient and its share of dA in LDS, per lane, its value at the starts
// of the blocks in the workspace.
template <typename T, bool GATED, int GROUPS>
__global__ __launch_bounds__(64 * Shape<GROUPS>::waves, 2) void k_packed_bwd(PackedScanArgs a)
{
    constexpr int WAVES = Shape<GROUPS>::waves;
    // Per wave: rows of values being folded (GROUPS > 1: then its sums over its states), gradients (forward: states), shares of dA, and
    // folded sums.  With 128 states that is all the LDS there is.
    constexpr int kRows = GROUPS > 1 ? 3 * kTok * 64 : 2 * kFoldRows, kKept = kStates * 64, kFolded = GROUPS == 1 ? kStates * 2 * kTok : 0;
    static_assert(kRows >= 2 * kFoldRows && kRows % 4 == 0 && kKept % 4 == 0 && kFolded % 4 == 0, "rows are read 16 bytes at a time");
    __shared__ __align__(16) float s_mem[WAVES][kRows + 2 * kKept + kFolded];
    static_assert(sizeof(s_mem) <= 160 * 1024, "a compute unit's LDS");
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
    const int n0 = GROUPS > 1 ? wave * kStates : 0;
    const int tile = (int)(blockIdx.x / (unsigned)a.groups), group = (int)(blockIdx.x % (unsigned)a.groups);
    const Piece p = a.ix.tiles[tile];
    if (!a.ix.good() || p.seq < 0) return;                       // (the same for every wave of the workgroup)
    int d = group * Shape<GROUPS>::channels + (GROUPS > 1 ? 0 : wave * 64) + lane;
    const bool on = d < a.D;
    if (!on) d = a.D - 1;                                        // lanes without a channel: another's inputs, no gradient
    const uint32_t off = (uint32_t)d * (uint32_t)sizeof(T);
    const int mine = min(kStates, a.N - n0);                     // this wave's states; none in a workgroup's last waves perhaps
    const int safe = mine > 0 ? n0 : 0;
    const float bias = a.bias ? a.bias[d] : 0.f, skip = a.Dv ? a.Dv[d] : 0.f;
    const bool sp = a.softplus != 0;
    const int64_t block0 = first_block(a.ix, p);
    const float* bc = a.bc + (block0 * 2 * a.N + safe) * 2 * kHalf;
    const int half = a.N * 2 * kHalf;                            // from one half of a block to the next
    const float* arow = a.A + (int64_t)d * a.N + safe;
    // where there is nothing to read (the sequence begins here, or the block is the tile's first) some finite value is read and counts 0:
    // a branch there would keep the compiler from asking early
    const float* some = reinterpret_cast<const float*>(a.ix.head);
    const bool begins = (p.bits & 1) != 0;                       // the sequence begins here, from zero
    const float* first_states = begins ? some : a.ends + ((int64_t)tile * a.N + safe) * a.D + d;
    const int64_t first_step = begins ? 0 : a.D;
    const float first_there = begins ? 0.f : 1.f;
    const int64_t slab = (int64_t)a.N * a.D;
    const int64_t starts_at = (int64_t)tile * (a.ix.tile / kTok - 1);
    const float* starts = a.starts + (starts_at * a.N + safe) * a.D + d;
    const float* start_sums = a.start_sums + starts_at * a.D + d;
    float* part = a.part_a + ((int64_t)tile * (a.N + 2) + safe) * a.D + d;
    float* rows = s_mem[wave];
    float* grads = rows + kRows + lane;
    float* shares = grads + kKept;
    constexpr int kFoldAt = kRows + 2 * kKept;
    const int blocks = (p.count + kTok - 1) / kTok;

    // The next block's tokens are asked for ahead of a block's loop over the states (forward) or of its last part (backward).
    Tokens<T, kTok> u, delta, dy, z;
    const auto request = [&](int b, int count) {
        const int64_t first = p.first + (int64_t)b * kTok;
        u = load_tokens<T, kTok>(Rows<T>(a.u, a.u_stride, first), count, off);
        delta = load_tokens<T, kTok>(Rows<T>(a.delta, a.d_stride, first), count, off);
    };
    const auto request_rest = [&](int b, int count) {
        const int64_t first = p.first + (int64_t)b * kTok;
        dy = load_tokens<T, kTok>(Rows<T>(a.dy, a.dy_stride, first), count, off);
        if constexpr (GATED) z = load_tokens<T, kTok>(Rows<T>(a.z, a.z_stride, first), count, off);
    };
    const int last_count = p.count - (blocks - 1) * kTok;
    request(blocks - 1, last_count);
    request_rest(blocks - 1, last_count);

#pragma unroll 4
    for (int n = 0; n < mine; ++n) {
        grads[n * 64] = on && !(p.bits & 2) ? a.backs[((int64_t)tile * a.N + safe + n) * a.D + d] : 0.f;
        shares[n * 64] = 0.f;
    }
    float dskip = 0.f, dbias = 0.f;
    for (int b = blocks - 1; b >= 0; --b) {
        const int64_t first = p.first + (int64_t)b * kTok;
        const int count = min(kTok, p.count - b * kTok);
        const int next = max(b - 1, 0), next_count = b > 0 ? kTok : count;       // (behind the first block: the same rows again, for nothing)
        float dl[kTok], dx[kTok], ds[kTok], gb[kTok], gk[kTok], out[kTok];
        const float* from = bc + (int64_t)b * 2 * half;
        // what a state's work takes from memory
        struct Ahead {
            float a, first, h;                                   // A, the tile's first state, the block's from zero
            State8 s[2];
        };
        const float* begin = b > 0 ? starts + (b - 1) * slab : some;
        const int64_t begin_step = b > 0 ? a.D : 0;
        const auto ask = [&](int n) {
            Ahead k;
            k.a = arow[n];
            k.first = first_states[n * first_step];
            k.h = begin[n * begin_step];
            k.s[0] = state8(from + n * 2 * kHalf);
            k.s[1] = state8(from + n * 2 * kHalf + half);
            return k;
        };
        Ahead even = ask(0), odd;
        if constexpr (GATED) gates<T, kTok>(z, ds);
        steps<T, kTok>(u, delta, bias, sp, count, dl, dx);
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            ds[t] = GATED ? ds[t] * dy.at(t) : dy.at(t);
            ds[t] = on && t < count ? ds[t] : 0.f;
            gb[t] = gk[t] = out[t] = 0.f;
        }
        const int64_t place = ((int64_t)group * a.blocks + block0 + b) * a.N + safe;
        const float before = b > 0 && !begins ? start_sums[(b - 1) * (int64_t)a.D] : 0.f, inside = b > 0 ? 1.f : 0.f;
        // a token's sums of dB and dC of state n: four lanes hold both, the even ones put the first in its place, the odd ones the second
        const auto put_fold = [&](int n, float sum_b, float sum_c) {
            const float sum = (lane & 1) ? sum_c : sum_b;
            const int spot = n * 2 * kTok + 2 * (lane >> 2) + (lane & 1);
            if constexpr (GROUPS == 1) s_mem[wave][kFoldAt + spot] = sum;
            else a.part_bc[place * 2 * kTok + spot] = sum;
        };
        // One state's work, which asks for the next one's values.
        const auto state = [&](int n, const Ahead& now, Ahead& next) {
            // What LDS has for this state and the folded rows of the one before are asked for ahead of the exponentials; behind them
            // comes the wait for all of it and for the scalar loads (they count together), and then the next scalar loads go out.
            const float a2 = rate(now.a);
            const float begun = first_there * now.first, own = inside * now.h;
            float h = begun == 0.f ? own : fmaf(fast_exp2(before * a2), begun, own), gn = grads[n * 64], an = shares[n * 64];
            const Quarter before_b = fold_read(rows, lane), before_c = fold_read(rows + kFoldRows, lane);
            float e[kTok], w[kTok], v[kTok];
#pragma unroll
            for (int t = 0; t < kTok; ++t) e[t] = dl[t] * a2;
            __builtin_amdgcn_sched_barrier(0);
            exp2_burst<kTok>(e);
            __builtin_amdgcn_sched_barrier(0);
            const State8 s[2] = {now.s[0], now.s[1]};
            put_fold(max(n - 1, 0), fold_sum(before_b), fold_sum(before_c));     // (of the first state: of what is there, overwritten by the next)
            next = ask(min(n + 1, mine - 1));
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < kTok; ++t) {
                w[t] = e[t] * h;                                 // a h_{t-1}
                h = fmaf(s[t / kHalf].b(t % kHalf), dx[t], w[t]);
                out[t] = fmaf(s[t / kHalf].c(t % kHalf), h, out[t]);
                v[t] = ds[t] * h;
            }
            fold_put(rows + kFoldRows, v, lane);
#pragma unroll
            for (int t = kTok - 1; t >= 0; --t) {
                gn = fmaf(s[t / kHalf].c(t % kHalf), ds[t], gn);
                gb[t] = fmaf(s[t / kHalf].b(t % kHalf), gn, gb[t]);
                const float through = gn * w[t];
                gk[t] = fmaf(a2, through, gk[t]);
                an = fmaf(dl[t], through, an);
                v[t] = gn * dx[t];
                gn *= e[t];
            }
            fold_put(rows, v, lane);
            grads[n * 64] = gn;
            shares[n * 64] = an;
        };
        // Two states a turn, so that what is asked for stays where it arrives: moved at the end of a turn it would be waited for there.
#pragma unroll 1
        for (int n = 0; n + 1 < mine; n += 2) {
            state(n, even, odd);
            state(n + 1, odd, even);
        }
        if (mine > 0 && (mine & 1)) state(mine - 1, even, odd);
        // what only the gate's gradient needs is read again (from the cache): kept, it would take the registers of a state's work
        if constexpr (GATED) request_rest(b, count);
        if (mine > 0) put_fold(mine - 1, fold_sum(fold_read(rows, lane)), fold_sum(fold_read(rows + kFoldRows, lane)));
        if constexpr (GROUPS == 1) {                             // dB and dC of the block, over the workgroup's channels
            __syncthreads();
            for (int i = (int)threadIdx.x; i < a.N * 2 * kTok; i += 64 * WAVES) {
                float sum = 0.f;
#pragma unroll
                for (int k = 0; k < WAVES; ++k) sum += s_mem[k][kFoldAt + i];
                a.part_bc[place * 2 * kTok + i] = sum;
            }
            __syncthreads();
        } else {                                                 // the sums over the waves' states; wave 0 finishes
            if (wave != 0) {
#pragma unroll
                for (int t = 0; t < kTok; ++t) {
                    rows[t * 64 + lane] = gb[t];
                    rows[(kTok + t) * 64 + lane] = gk[t];
                    rows[(2 * kTok + t) * 64 + lane] = out[t];
                }
            }
            __syncthreads();
            if (wave == 0) {
                for (int k = 1; k < GROUPS; ++k) {
#pragma unroll
                    for (int t = 0; t < kTok; ++t) {
                        gb[t] += s_mem[k][t * 64 + lane];
                        gk[t] += s_mem[k][(kTok + t) * 64 + lane];
                        out[t] += s_mem[k][(2 * kTok + t) * 64 + lane];
                    }
                }
            }
            __syncthreads();
            if (wave != 0) {
                request(next, next_count);
                request_rest(next, next_count);
                continue;
            }
        }
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            gk[t] = fmaf(u.at(t), gb[t], gk[t] * kLn2);
            gb[t] = fmaf(skip, ds[t], dl[t] * gb[t]);
            dskip = fmaf(ds[t], u.at(t), dskip);                 // (ds is 0 for tokens that are not there)
            out[t] = fmaf(skip, u.at(t), out[t]);
        }
        float sig[kTok];
#pragma unroll
        for (int t = 0; t < kTok; ++t) sig[t] = -(delta.at(t) + bias) * kLog2e;
        request(next, next_count);
        if (on) store_tokens<T, kTok>(Rows<T>(a.du, a.du_stride, first), count, off, gb);
        if (sp) {                                                // times sigmoid(delta + bias)
            exp2_burst<kTok>(sig);
#pragma unroll
            for (int t = 0; t < kTok; ++t) sig[t] += 1.f;
            rcp_burst<kTok>(sig);
#pragma unroll
            for (int t = 0; t < kTok; ++t) gk[t] *= sig[t];
        }
#pragma unroll
        for (int t = 0; t < kTok; ++t) dbias += t < count ? gk[t] : 0.f;
        if (on) store_tokens<T, kTok>(Rows<T>(a.ddelta, a.dd_stride, first), count, off, gk);
        if constexpr (GATED) {
#pragma unroll
            for (int t = 0; t < kTok; ++t) sig[t] = -z.at(t) * kLog2e;
            exp2_burst<kTok>(sig);
#pragma unroll
            for (int t = 0; t < kTok; ++t) sig[t] += 1.f;
            rcp_burst<kTok>(sig);
#pragma unroll
            for (int t = 0; t < kTok; ++t) out[t] *= dy.at(t) * (sig[t] * fmaf(z.at(t), 1.f - sig[t], 1.f));
            request_rest(next, next_count);
            if (on) store_tokens<T, kTok>(Rows<T>(a.dz, a.dz_stride, first), count, off, out);
        } else {
            request_rest(next, next_count);
        }
    }
    if (!on) return;
    for (int n = 0; n < mine; ++n) part[(int64_t)n * a.D] = shares[n * 64];
    if (n0 != 0) return;
    part[(int64_t)a.N * a.D] = dskip;
    part[(int64_t)(a.N + 1) * a.D] = dbias;
}

// dB and dC: the workgroups' sums.  A lane takes one token and state of one of them.
template <typename T> __global__ __launch_bounds__(256) void k_packed_bwd_bc(PackedScanArgs a)
{
    const int64_t per = 2 * kTok * a.N, i = (int64_t)blockIdx.x * 256 + threadIdx.x, block = i / per;
    if (block >= a.blocks || !a.ix.good()) return;
    const Piece p = a.ix.blocks[block];
    const int j = (int)(i - block * per), t = (j >> 1) & (kTok - 1), n = j / (2 * kTok);
    if (p.seq < 0 || t >= p.count) return;
    float sum = 0.f;
    for (int g = 0; g < a.groups; ++g) sum += a.part_bc[(int64_t)g * a.blocks * per + i];
    if (j & 1) Io<T>::st(static_cast<T*>(a.dC) + (p.first + (int64_t)t) * a.dc_stride + n, sum);
    else Io<T>::st(static_cast<T*>(a.dB) + (p.first + (int64_t)t) * a.db_stride + n, sum);
}

// dA, dD, dbias: the tiles' sums.  A workgroup takes 64 columns; its waves the tiles in turn.
__global__ __launch_bounds__(256) void k_packed_bwd_a(PackedScanArgs a)
{
    __shared__ float part[4][64];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int64_t n = (int64_t)(a.N + 2) * a.D, col = (int64_t)blockIdx.x * 64 + lane;
    float s[4] = {};
    if (col < n && a.ix.good()) {
        const int tiles = a.ix.head[5];
        int k = wave;
        for (; k + 12 < tiles; k += 16) {
#pragma unroll
            for (int q = 0; q < 4; ++q) s[q] += a.part_a[(k + 4 * q) * n + col];
        }
        for (; k < tiles; k += 4) s[0] += a.part_a[k * n + col];
    }
    part[wave][lane] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (wave != 0 || col >= n || !a.ix.good()) return;
    const float sum = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
    const int row = (int)(col / a.D), d = (int)(col % a.D);
    if (row < a.N) a.dA[(int64_t)d * a.N + row] = sum;
    else if (row == a.N) {
        if (a.dD) a.dD[d] = sum;
    } else if (a.dbias) {
        a.dbias[d] = sum;
    }
}

// The workspace's parts, in floats.
struct Space {
    int64_t bc, ends, backs, sums, starts, start_sums, part_bc, part_a, all;
};
Space space(const Layout& l, int64_t T, int32_t tile, int64_t D, int64_t N)
{
    const int64_t tiles = T > tile ? l.max_tiles : 0;            // (carried only where a sequence can have a second tile)
    const int64_t groups = channel_groups(D, N);
    Space s;
    s.bc = 0;
    s.ends = s.bc + l.max_blocks * N * 32 + 48;                  // (the loop over the states asks for three more than there are)
    s.backs = s.ends + tiles * N * D;
    s.sums = s.backs + tiles * N * D;
    s.starts = s.sums + tiles * D;
    s.start_sums = s.starts + l.max_tiles * (tile / kTok - 1) * N * D;
    s.part_bc = s.start_sums + l.max_tiles * (tile / kTok - 1) * D;
    s.part_a = s.part_bc + groups * l.max_blocks * 32 * N;
    s.all = s.part_a + l.max_tiles * (N + 2) * D;
    return s;
}

}  // namespace

extern "C" size_t corey_scan_packed_bwd_workspace(const corey_pack* pack, int64_t D, int64_t N)
{
    Index ix;
    if (D < 1 || D > COREY_PACK_MAX_CHANNELS || N < 1 || N > COREY_PACK_MAX_STATE || index_of("corey_scan_packed_bwd_workspace", pack, &ix)) return 0;
    return (size_t)space(layout(pack->S, pack->T, pack->tile), pack->T, pack->tile, D, N).all * 4;
}

extern "C" int corey_scan_packed_bwd(const void* u, int64_t u_stride, const void* delta, int64_t delta_stride, const float* A,
                                     const void* Bm, int64_t B_stride, const void* Cm, int64_t C_stride, const float* Dv, const void* z,
                                     int64_t z_stride, const float* delta_bias, int delta_softplus, const void* dy, int64_t dy_stride,
                                     const corey_pack* pack, void* du, int64_t du_stride, void* ddelta, int64_t ddelta_stride, float* dA,
                                     void* dB, int64_t dB_stride, void* dC, int64_t dC_stride, float* dDv, void* dz, int64_t dz_stride,
                                     float* ddelta_bias, corey_dtype dt, int64_t D, int64_t N, void* workspace, size_t workspace_bytes,
                                     void* hip_stream)
{
    using corey::fail;
    const char* who = "corey_scan_packed_bwd";
    if (!u || !delta || !A || !Bm || !Cm || !dy || !du || !ddelta || !dA || !dB || !dC)
        return fail(COREY_ENULL, "%s: u, delta, A, Bm, Cm, dy, du, ddelta, dA, dB and dC are required", who);
    if ((z != nullptr) != (dz != nullptr)) return fail(COREY_ENULL, "%s: dz goes with z", who);
    if (!good_dtype(dt)) return fail(COREY_EINVAL, "%s: unknown dtype %d", who, (int)dt);
    if (D < 1 || D > COREY_PACK_MAX_CHANNELS || N < 1) return fail(COREY_ESHAPE, "%s: 1 <= D <= %d and N >= 1 required", who, COREY_PACK_MAX_CHANNELS);
    if (N > COREY_PACK_MAX_STATE) return fail(COREY_EUNSUPPORTED, "%s: N above %d", who, COREY_PACK_MAX_STATE);
    if (!good_stride(u_stride, D) || !good_stride(delta_stride, D) || !good_stride(dy_stride, D) || !good_stride(du_stride, D) ||
        !good_stride(ddelta_stride, D) || (z && (!good_stride(z_stride, D) || !good_stride(dz_stride, D))) || !good_stride(B_stride, N) ||
        !good_stride(C_stride, N) || !good_stride(dB_stride, N) || !good_stride(dC_stride, N))
        return fail(COREY_ESHAPE, "%s: rows must be at least D (B, C and their gradients: N) apart", who);
    const void* ins[] = {u, delta, Bm, Cm, z, dy};
    const void* outs[] = {du, ddelta, dB, dC, dz};
    for (size_t i = 0; i < 5; ++i) {
        for (const void* in : ins)
            if (outs[i] && outs[i] == in) return fail(COREY_EINVAL, "%s: a gradient may not be an input", who);
        for (size_t j = 0; j < i; ++j)
            if (outs[i] && outs[i] == outs[j]) return fail(COREY_EINVAL, "%s: two gradients in one place", who);
    }
    PackedScanArgs a = {};
    if (int e = index_of(who, pack, &a.ix)) return e;
    if (pack->tile > kMaxBackTile || (N > 64 && pack->tile > 32))
        return fail(COREY_EUNSUPPORTED, "%s: the index's tile must be at most 64, and 32 for N > 64", who);
    const Layout l = layout(pack->S, pack->T, pack->tile);
    const Space w = space(l, pack->T, pack->tile, D, N);
    if (!workspace || workspace_bytes < (size_t)w.all * 4 || reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
        return fail(COREY_EWORKSPACE, "%s: workspace missing, misaligned or smaller than corey_scan_packed_bwd_workspace()", who);
    float* ws = static_cast<float*>(workspace);
    a.u = u; a.delta = delta; a.Bm = Bm; a.Cm = Cm; a.z = z; a.dy = dy;
    a.A = A; a.Dv = Dv; a.bias = delta_bias;
    a.u_stride = u_stride; a.d_stride = delta_stride; a.b_stride = B_stride; a.c_stride = C_stride; a.z_stride = z_stride; a.dy_stride = dy_stride;
    a.du = du; a.ddelta = ddelta; a.dz = dz; a.dB = dB; a.dC = dC;
    a.du_stride = du_stride; a.dd_stride = ddelta_stride; a.dz_stride = dz_stride; a.db_stride = dB_stride; a.dc_stride = dC_stride;
    a.dA = dA; a.dD = dDv; a.dbias = ddelta_bias;
    a.bc = ws + w.bc; a.ends = ws + w.ends; a.backs = ws + w.backs; a.sums = ws + w.sums; a.starts = ws + w.starts; a.start_sums = ws + w.start_sums; a.part_bc = ws + w.part_bc; a.part_a = ws + w.part_a;
    a.D = (int32_t)D; a.N = (int32_t)N;
    a.softplus = delta_softplus ? 1 : 0;
    a.blocks = (int32_t)l.max_blocks;
    a.groups = (int32_t)channel_groups(D, N);
    const int64_t columns = (D * N + 255) / 256, groups = channel_groups(D, N);
    const int64_t relay = (l.max_blocks * N * 32 + 255) / 256;
    if (!good_grid(l.max_tiles * groups, 64 * waves_of(N)) || !good_grid(2 * columns * l.max_longs, 256) || !good_grid(relay, 256))
        return fail(COREY_ESHAPE, "%s: T * D is too large", who);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    by_type(dt, [&](auto t) {
        using T = decltype(t);
        by_groups(N, [&](auto gr) {
            constexpr int G = decltype(gr)::value;
            const auto go = [&](auto gate, auto whole) {
                constexpr bool Z = decltype(gate)::value;
                k_packed_relay<T><<<(unsigned)relay, 256, 0, stream>>>(a);
                if (pack->T > kTok) k_packed_bwd_ends<T, Z, G, decltype(whole)::value><<<(unsigned)(l.max_tiles * groups), 64 * Shape<G>::waves, 0, stream>>>(a);
                if (pack->T > pack->tile) k_packed_bwd_chain<<<(unsigned)(2 * columns * l.max_longs), 256, 0, stream>>>(a, (int)columns);
                k_packed_bwd<T, Z, G><<<(unsigned)(l.max_tiles * groups), 64 * Shape<G>::waves, 0, stream>>>(a);
            };
            const auto with = [&](auto gate) {
                if (N == G * kStates) go(gate, std::true_type());
                else go(gate, std::false_type());
            };
            if (z) with(std::true_type());
            else with(std::false_type());
        });
        k_packed_bwd_bc<T><<<(unsigned)relay, 256, 0, stream>>>(a);
    });
    k_packed_bwd_a<<<(unsigned)(((N + 2) * D + 63) / 64), 256, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? corey::hip_fail(e, "corey_scan_packed_bwd launch") : COREY_OK;
}
