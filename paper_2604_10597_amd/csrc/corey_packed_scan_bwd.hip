// corey_scan_packed_bwd: the gradients of the selective scan on packed batches, from dy and the scan's inputs.
//
//     a_t = exp(dl_t A), h_t = a_t h_{t-1} + dl_t B_t u_t, s_t = sum_n C_t h_t + D u_t, y_t = s_t silu(z_t);   ds = dy silu(z)
//     g_t = ds_t C_t + a_{t+1} g_{t+1}                        (the gradient of h_t)
//     dC_t = sum_d ds h,  dB_t = sum_d g dl u,  ddl = sum_n g (u B + A a h_{t-1}),  du = D ds + dl sum_n g B,  dA = sum_t g dl a h_{t-1}
//
// Sequences are cut into tiles of at most 64 tokens that are walked side by side:
//   k_packed_bwd_ends   every tile of a longer sequence: its end state E from zero, the gradient G that it hands to the state it begins
//                       with when none comes from behind, and the sum of its step sizes
//   k_packed_bwd_chain  per sequence, over its tiles: forward h_k+1 = exp(A sum) h_k + E_k, backward g_k-1 = exp(A sum) g_k + G_k
//   k_packed_bwd        every tile: the states at the starts of its blocks of 16 tokens (kept in LDS), then block by block from the
//                       last, state by state: the block's decays and states forward, its gradients backward.  Sums over states stay
//                       in the lane (a lane is a channel); sums over channels (dB, dC) are folded over the wave's lanes, over the
//                       workgroup's waves in LDS, and written per workgroup
//   k_packed_bwd_bc, k_packed_bwd_a   add up the workgroups' dB and dC, and the tiles' dA, dD and dbias, always in the same order
// Per token, channel and state: three exponentials and some 35 plain instructions; vector issue is the bound.
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
    if (!a.ix.good() || p.seq < 0 || p.bits == 3 || n0 >= a.N) return;
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
        a2[n] *= kLog2e;
        h[n] = back[n] = 0.f;
    }
    const float bias = a.bias ? a.bias[d] : 0.f;
    const float* from = a.bc + (first_block(a.ix, p) * 2 * a.N + n0) * 2 * kHalf;
    for (int t0 = 0; t0 < p.count; t0 += K) {
        const int count = p.count - t0;
        State8 s[3];                                             // two states ahead
        s[0] = state8(from);
        s[1] = state8(from + 2 * kHalf);
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
            if (n + 2 < kStates) s[(n + 2) % 3] = state8(from + (n + 2) * 2 * kHalf);   // (behind the last: the next block's, or the end's)
            float e[K], x[K], g = 0.f;
            arguments<K>(dl, a2[n], dx, [&](int t) { return s[n % 3].b(t); }, e, x);
#pragma unroll
            for (int t = 0; t < K; ++t) {
                h[n] = fmaf(e[t], h[n], x[t]);
                const int r = K - 1 - t;                         // (and the gradients from the last token back)
                g = fmaf(s[n % 3].c(r), ds[r], g) * e[r];
            }
            back[n] = fmaf(fast_exp2(before * a2[n]), g, back[n]);
            __builtin_amdgcn_sched_barrier(0);
        }
        from += a.N * 2 * kHalf;
    }
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
    const float a2 = a.A[(int64_t)d * a.N + n] * kLog2e;
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
                h = fmaf(fast_exp2(a2 * sum[i]), h, end[i]);
            }
        }
    }
}

// 16 values of every lane, summed over the wave's 64 lanes: every lane leaves with the sum of value lane / 4.  Halving: lanes of one
// half hand over the values that the other half sums.  Across 32 and 16 lanes the swap instructions bring both halves' parts of two
// values into place at once; below, DPP.
__device__ __forceinline__ float fold16(float (&v)[16], int lane)
{
    auto swap_add = [](float& x, float y, auto swap) {
        const auto r = swap(__float_as_uint(x), __float_as_uint(y));
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    };
#pragma unroll
    for (int i = 0; i < 8; ++i) swap_add(v[i], v[i + 8], [](uint32_t x, uint32_t y) { return __builtin_amdgcn_permlane32_swap(x, y, false, false); });
#pragma unroll
    for (int i = 0; i < 4; ++i) swap_add(v[i], v[i + 4], [](uint32_t x, uint32_t y) { return __builtin_amdgcn_permlane16_swap(x, y, false, false); });
    constexpr int kXor8 = 0x128, kMirror8 = 0x141, kXor2 = 0x4e, kXor1 = 0xb1;     // row_ror:8, row_half_mirror, quad_perm
    const bool b3 = (lane & 8) != 0, b2 = (lane & 4) != 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float keep = b3 ? v[i + 2] : v[i], send = b3 ? v[i] : v[i + 2];
        v[i] = keep + dpp_move<kXor8>(send);
    }
    const float keep = b2 ? v[1] : v[0], send = b2 ? v[0] : v[1];
    float r = keep + dpp_move<kMirror8>(send);
    r += dpp_move<kXor2>(r);
    r += dpp_move<kXor1>(r);
    return r;
}

// Values of a wave's states that it keeps in LDS, per lane: at the starts of blocks 1, 2, ... (a slot each), and the gradients.
__host__ __device__ constexpr int kept(int tile) { return tile / kTok; }

// The loop over the states is a loop (unrolled it is 50 KB of instructions, more than the instruction cache feeds), so what belongs to
// a state from block to block stays out of registers: its value at the starts of the blocks and its gradient in LDS, its share of dA
// in the workspace, where each lane adds to its own.
template <typename T, bool GATED, int GROUPS>
__global__ __launch_bounds__(64 * Shape<GROUPS>::waves, 2) void k_packed_bwd(PackedScanArgs a)
{
    constexpr int WAVES = Shape<GROUPS>::waves;
    __shared__ float s_fold[GROUPS == 1 ? WAVES : 1][GROUPS == 1 ? kStates * 2 * kTok : 1];
    __shared__ float s_part[GROUPS > 1 ? GROUPS - 1 : 1][GROUPS > 1 ? 3 * kTok * 64 : 1];
    extern __shared__ float s_kept[];     // [WAVES][kept(tile)][16 states][64 lanes]
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
    const float* first_states = a.ends + ((int64_t)tile * a.N + safe) * a.D + d;
    float* part = a.part_a + ((int64_t)tile * (a.N + 2) + safe) * a.D + d;
    const bool begins = (p.bits & 1) != 0;                       // the sequence begins here, from zero
    float* starts = s_kept + (int64_t)wave * kept(a.ix.tile) * kStates * 64 + lane;
    float* grads = starts + (kept(a.ix.tile) - 1) * kStates * 64;
    const int blocks = (p.count + kTok - 1) / kTok;
    // a state at the start of block b
    const auto start_of = [&](int b, int n) {
        if (b > 0) return starts[((b - 1) * kStates + n) * 64];
        return begins ? 0.f : first_states[(int64_t)n * a.D];
    };

    // forward over all blocks but the last: the states that blocks 1, 2, ... begin with
    for (int b = 0; b + 1 < blocks; ++b) {
        float dl[kTok], dx[kTok];
        const int64_t first = p.first + (int64_t)b * kTok;
        const float* from = bc + (int64_t)b * 2 * half;
        float a_next = arow[0], h_next = start_of(b, 0);
        State8 s_next[2] = {state8(from), state8(from + half)};
        steps<T, kTok>(load_tokens<T, kTok>(Rows<T>(a.u, a.u_stride, first), kTok, off), load_tokens<T, kTok>(Rows<T>(a.delta, a.d_stride, first), kTok, off),
                       bias, sp, kTok, dl, dx);
#pragma unroll 1
        for (int n = 0; n < mine; ++n) {
            const float a2 = a_next * kLog2e;
            float h = h_next;
            const State8 s[2] = {s_next[0], s_next[1]};
            const int m = min(n + 1, mine - 1);
            a_next = arow[m];
            h_next = start_of(b, m);
            s_next[0] = state8(from + m * 2 * kHalf);
            s_next[1] = state8(from + m * 2 * kHalf + half);
            float e[kTok], x[kTok];
            arguments<kTok>(dl, a2, dx, [&](int t) { return s[t / kHalf].b(t % kHalf); }, e, x);
#pragma unroll
            for (int t = 0; t < kTok; ++t) h = fmaf(e[t], h, x[t]);
            starts[(b * kStates + n) * 64] = h;
        }
    }

    for (int n = 0; n < mine; ++n)
        grads[n * 64] = on && !(p.bits & 2) ? a.backs[((int64_t)tile * a.N + safe + n) * a.D + d] : 0.f;
    float dskip = 0.f, dbias = 0.f;
    for (int b = blocks - 1; b >= 0; --b) {
        const int64_t first = p.first + (int64_t)b * kTok;
        const int count = min(kTok, p.count - b * kTok);
        float dl[kTok], dx[kTok], ds[kTok], gb[kTok], gk[kTok], out[kTok];
        const float* from = bc + (int64_t)b * 2 * half;
        State8 s_next[2] = {state8(from), state8(from + half)};
        {
            const Tokens<T, kTok> u = load_tokens<T, kTok>(Rows<T>(a.u, a.u_stride, first), count, off),
                                  delta = load_tokens<T, kTok>(Rows<T>(a.delta, a.d_stride, first), count, off),
                                  dy = load_tokens<T, kTok>(Rows<T>(a.dy, a.dy_stride, first), count, off);
            if constexpr (GATED) gates<T, kTok>(load_tokens<T, kTok>(Rows<T>(a.z, a.z_stride, first), count, off), ds);
            steps<T, kTok>(u, delta, bias, sp, count, dl, dx);
#pragma unroll
            for (int t = 0; t < kTok; ++t) {
                ds[t] = GATED ? ds[t] * dy.at(t) : dy.at(t);
                ds[t] = on && t < count ? ds[t] : 0.f;
                gb[t] = gk[t] = out[t] = 0.f;
            }
        }
        const int64_t place = ((int64_t)group * a.blocks + block0 + b) * a.N + safe;
        const bool fresh = b == blocks - 1;
        float a_next = arow[0], h_next = start_of(b, 0);
#pragma unroll 1
        for (int n = 0; n < mine; ++n) {
            const float a2 = a_next * kLog2e;
            float h = h_next, gn = grads[n * 64], an = fresh ? 0.f : part[(int64_t)n * a.D];
            const State8 s[2] = {s_next[0], s_next[1]};
            const int m = min(n + 1, mine - 1);
            a_next = arow[m];
            h_next = start_of(b, m);
            s_next[0] = state8(from + m * 2 * kHalf);
            s_next[1] = state8(from + m * 2 * kHalf + half);
            float e[kTok], w[kTok], v[kTok];
            arguments<kTok>(dl, a2, dx, [&](int t) { return s[t / kHalf].b(t % kHalf); }, e, v);
#pragma unroll
            for (int t = 0; t < kTok; ++t) {
                w[t] = e[t] * h;                                 // a h_{t-1}
                h = w[t] + v[t];
                out[t] = fmaf(s[t / kHalf].c(t % kHalf), h, out[t]);
                v[t] = ds[t] * h;
            }
            const float sum_c = fold16(v, lane);
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
            const float sum_b = fold16(v, lane);
            const float folded = (lane & 1) ? sum_c : sum_b;     // (two lanes each hold the same value for the same place)
            const int spot = n * 2 * kTok + 2 * (lane >> 2) + (lane & 1);
            if constexpr (GROUPS == 1) s_fold[wave][spot] = folded;
            else a.part_bc[place * 2 * kTok + spot] = folded;
            grads[n * 64] = gn;
            if (on) part[(int64_t)n * a.D] = an;
        }
        if constexpr (GROUPS == 1) {                             // dB and dC of the block, over the workgroup's channels
            __syncthreads();
            for (int i = (int)threadIdx.x; i < a.N * 2 * kTok; i += 64 * WAVES) {
                float sum = 0.f;
#pragma unroll
                for (int k = 0; k < WAVES; ++k) sum += s_fold[k][i];
                a.part_bc[place * 2 * kTok + i] = sum;
            }
            __syncthreads();
        } else {                                                 // the sums over the waves' states; wave 0 finishes
            __syncthreads();
            if (wave != 0) {
#pragma unroll
                for (int t = 0; t < kTok; ++t) {
                    s_part[wave - 1][t * 64 + lane] = gb[t];
                    s_part[wave - 1][(kTok + t) * 64 + lane] = gk[t];
                    s_part[wave - 1][(2 * kTok + t) * 64 + lane] = out[t];
                }
            }
            __syncthreads();
            if (wave != 0) continue;
            for (int k = 0; k + 1 < GROUPS; ++k) {
#pragma unroll
                for (int t = 0; t < kTok; ++t) {
                    gb[t] += s_part[k][t * 64 + lane];
                    gk[t] += s_part[k][(kTok + t) * 64 + lane];
                    out[t] += s_part[k][(2 * kTok + t) * 64 + lane];
                }
            }
        }
        // what only the end needs is read again (from the cache): kept, it would take the registers of a state's work
        const Tokens<T, kTok> u = load_tokens<T, kTok>(Rows<T>(a.u, a.u_stride, first), count, off),
                              delta = load_tokens<T, kTok>(Rows<T>(a.delta, a.d_stride, first), count, off);
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            gk[t] = fmaf(u.at(t), gb[t], gk[t] * kLn2);
            gb[t] = fmaf(skip, ds[t], dl[t] * gb[t]);
            dskip = fmaf(ds[t], u.at(t), dskip);                 // (ds is 0 for tokens that are not there)
            out[t] = fmaf(skip, u.at(t), out[t]);
        }
        if (on) store_tokens<T, kTok>(Rows<T>(a.du, a.du_stride, first), count, off, gb);
        if (sp) {                                                // times sigmoid(delta + bias)
            float sig[kTok];
#pragma unroll
            for (int t = 0; t < kTok; ++t) sig[t] = -(delta.at(t) + bias) * kLog2e;
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
            const Tokens<T, kTok> z = load_tokens<T, kTok>(Rows<T>(a.z, a.z_stride, first), count, off),
                                  dy = load_tokens<T, kTok>(Rows<T>(a.dy, a.dy_stride, first), count, off);
            float sig[kTok];
#pragma unroll
            for (int t = 0; t < kTok; ++t) sig[t] = -z.at(t) * kLog2e;
            exp2_burst<kTok>(sig);
#pragma unroll
            for (int t = 0; t < kTok; ++t) sig[t] += 1.f;
            rcp_burst<kTok>(sig);
#pragma unroll
            for (int t = 0; t < kTok; ++t) out[t] *= dy.at(t) * (sig[t] * fmaf(z.at(t), 1.f - sig[t], 1.f));
            if (on) store_tokens<T, kTok>(Rows<T>(a.dz, a.dz_stride, first), count, off, out);
        }
    }
    if (!on || n0 != 0) return;
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
    int64_t bc, ends, backs, sums, part_bc, part_a, all;
};
Space space(const Layout& l, int64_t T, int32_t tile, int64_t D, int64_t N)
{
    const int64_t tiles = T > tile ? l.max_tiles : 0;            // (carried only where a sequence can have a second tile)
    const int64_t groups = channel_groups(D, N);
    Space s;
    s.bc = 0;
    s.ends = s.bc + l.max_blocks * N * 32 + 32;                  // (the loop over the states asks for one more than there is)
    s.backs = s.ends + tiles * N * D;
    s.sums = s.backs + tiles * N * D;
    s.part_bc = s.sums + tiles * D;
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
    a.bc = ws + w.bc; a.ends = ws + w.ends; a.backs = ws + w.backs; a.sums = ws + w.sums; a.part_bc = ws + w.part_bc; a.part_a = ws + w.part_a;
    a.D = (int32_t)D; a.N = (int32_t)N;
    a.softplus = delta_softplus ? 1 : 0;
    a.blocks = (int32_t)l.max_blocks;
    a.groups = (int32_t)channel_groups(D, N);
    const int64_t columns = (D * N + 255) / 256, groups = channel_groups(D, N);
    const int64_t relay = (l.max_blocks * N * 32 + 255) / 256;
    if (l.max_tiles * groups > INT32_MAX || 2 * columns * (l.max_longs + 1) > INT32_MAX || relay > INT32_MAX)
        return fail(COREY_ESHAPE, "%s: T * D is too large", who);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    hipError_t attr = hipSuccess;
    by_type(dt, [&](auto t) {
        using T = decltype(t);
        by_groups(N, [&](auto gr) {
            constexpr int G = decltype(gr)::value;
            const auto go = [&](auto gate, auto whole) {
                constexpr bool Z = decltype(gate)::value;
                const size_t lds = (size_t)Shape<G>::waves * (size_t)kept(pack->tile) * kStates * 64 * 4;
                // (what the longest tile takes, whatever this call's: another thread's call may be between this line and its launch)
                constexpr int most = Shape<G>::waves * kept(G == 8 ? 32 : kMaxBackTile) * kStates * 64 * 4;
                attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_packed_bwd<T, Z, G>), hipFuncAttributeMaxDynamicSharedMemorySize, most);
                if (attr != hipSuccess) return;
                k_packed_relay<T><<<(unsigned)relay, 256, 0, stream>>>(a);
                if (pack->T > pack->tile) {
                    k_packed_bwd_ends<T, Z, G, decltype(whole)::value><<<(unsigned)(l.max_tiles * groups), 64 * Shape<G>::waves, 0, stream>>>(a);
                    k_packed_bwd_chain<<<(unsigned)(2 * columns * l.max_longs), 256, 0, stream>>>(a, (int)columns);
                }
                k_packed_bwd<T, Z, G><<<(unsigned)(l.max_tiles * groups), 64 * Shape<G>::waves, lds, stream>>>(a);
            };
            const auto with = [&](auto gate) {
                if (N == G * kStates) go(gate, std::true_type());
                else go(gate, std::false_type());
            };
            if (z) with(std::true_type());
            else with(std::false_type());
        });
        if (attr == hipSuccess) k_packed_bwd_bc<T><<<(unsigned)relay, 256, 0, stream>>>(a);
    });
    if (attr != hipSuccess) return corey::hip_fail(attr, "corey_scan_packed_bwd: LDS");
    k_packed_bwd_a<<<(unsigned)(((N + 2) * D + 63) / 64), 256, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? corey::hip_fail(e, "corey_scan_packed_bwd launch") : COREY_OK;
}
