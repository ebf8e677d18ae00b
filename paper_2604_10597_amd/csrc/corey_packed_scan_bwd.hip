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

constexpr int kTok = 16;                  // tokens of a block
constexpr int kMaxBackTile = 64;

template <typename T, bool NEIGHBOURS, bool GATED, int GROUPS>
__global__ __launch_bounds__(64 * GROUPS, 2) void k_packed_bwd_ends(PackedScanArgs a)
{
    __shared__ __align__(16) float s_b[GROUPS][2][kStates * K], s_c[GROUPS][2][kStates * K];
    const int wave = GROUPS > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : 0, lane = (int)threadIdx.x & 63;
    const int n0 = wave * kStates;
    const int tile = (int)(blockIdx.x / (unsigned)a.groups);
    const Piece p = a.ix.tiles[tile];
    if (!a.ix.good() || p.seq < 0 || p.bits == 3 || n0 >= a.N) return;
    const Channels<NEIGHBOURS> c((int)(blockIdx.x % (unsigned)a.groups), lane, a.D);
    States s;
    load_a(s, a.A, c.d, n0, a.N);
    float bias[2], sum[2] = {}, back[kStates][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) bias[i] = a.bias ? a.bias[c.d[i]] : 0.f;
#pragma unroll
    for (int n = 0; n < kStates; ++n) {
#pragma unroll
        for (int i = 0; i < 2; ++i) s.h[n][i] = back[n][i] = 0.f;
    }
    Block<T> now;
    request<T, true, GATED, true>(now, a, c, n0, p.first, p.count);
    int buf = 0;
    for (int t0 = 0; t0 < p.count; t0 += K, buf ^= 1) {
        float dl[2 * K], dx[2 * K], ds[2 * K];
        const int count = p.count - t0;
        float* sb = s_b[wave][buf];
        float* sc = s_c[wave][buf];
        stage<T, true>(now, sb, sc);
        steps<T>(now, bias, a.softplus != 0, count, dl, dx, ds);
#pragma unroll
        for (int i = 0; i < 2 * K; ++i) {
            ds[i] = Io<T>::ld(&now.dy[i / 2].v[i & 1]);
            if constexpr (GATED) ds[i] *= silu(Io<T>::ld(&now.z[i / 2].v[i & 1]));
            ds[i] = i / 2 < count ? ds[i] : 0.f;
        }
        const float before[2] = {sum[0], sum[1]};               // the decay up to this block is exp(A before)
#pragma unroll
        for (int i = 0; i < 2 * K; ++i) sum[i & 1] += dl[i];
        if (t0 + K < p.count) request<T, true, GATED, true>(now, a, c, n0, p.first + t0 + K, count - K);
        lds_in_order();
        Words<K> bv[2], cv[2];
        bv[0] = words<K>(sb);
        cv[0] = words<K>(sc);
#pragma unroll
        for (int n = 0; n < kStates; ++n) {
            if (n + 1 < kStates) {
                bv[(n + 1) & 1] = words<K>(sb + (n + 1) * K);
                cv[(n + 1) & 1] = words<K>(sc + (n + 1) * K);
            }
            float d[2 * K];
#pragma unroll
            for (int i = 0; i < 2 * K; ++i) d[i] = dl[i] * s.a2[n][i & 1];
            exp2_burst<2 * K>(d);
#pragma unroll
            for (int t = 0; t < K; ++t) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    s.h[n][i] = fmaf(d[2 * t + i], s.h[n][i], dx[2 * t + i] * bv[n & 1].v[t]);
                }
            }
            float g[2] = {};
#pragma unroll
            for (int t = K - 1; t >= 0; --t) {
#pragma unroll
                for (int i = 0; i < 2; ++i) g[i] = fmaf(ds[2 * t + i], cv[n & 1].v[t], g[i]) * d[2 * t + i];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) back[n][i] = fmaf(fast_exp2(before[i] * s.a2[n][i]), g[i], back[n][i]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    const int64_t at = ((int64_t)tile * a.N + n0) * a.D;
#pragma unroll
    for (int n = 0; n < kStates; ++n) {
        if (n0 + n < a.N) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (!c.on[i]) continue;
                a.ends[at + (int64_t)n * a.D + c.d[i]] = s.h[n][i];
                a.backs[at + (int64_t)n * a.D + c.d[i]] = back[n][i];
            }
        }
    }
    if (wave == 0) {
        if (c.on[0]) a.sums[(int64_t)tile * a.D + c.d[0]] = sum[0];
        if (c.on[1]) a.sums[(int64_t)tile * a.D + c.d[1]] = sum[1];
    }
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

// Waves of a workgroup: the channels' for up to 16 states (4 x 64 channels), the states' otherwise (64 channels).
template <int GROUPS> constexpr int channel_waves() { return GROUPS == 1 ? 4 : 1; }
template <int GROUPS> constexpr int back_waves() { return GROUPS * channel_waves<GROUPS>(); }
__host__ __device__ constexpr int start_slots(int tile) { return tile > kTok ? tile / kTok - 1 : 1; }
constexpr int kFold = 33;                 // floats of a state's folded sums in LDS: 16 tokens x (dB, dC), and one against bank conflicts

template <typename T, bool GATED, int GROUPS>
__global__ __launch_bounds__(64 * back_waves<GROUPS>(), 2) void k_packed_bwd(PackedScanArgs a)
{
    constexpr int CW = channel_waves<GROUPS>(), WAVES = back_waves<GROUPS>();
    __shared__ __align__(16) float s_b[WAVES][kStates * kTok], s_c[WAVES][kStates * kTok];
    __shared__ float s_fold[WAVES][kStates * kFold];
    __shared__ float s_part[GROUPS > 1 ? GROUPS - 1 : 1][GROUPS > 1 ? 3 * kTok * 64 : 1];
    extern __shared__ float s_starts[];   // [WAVES][slots][16 states][64 lanes]: states at the starts of blocks 1, 2, ...
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
    const int n0 = GROUPS > 1 ? wave * kStates : 0;
    const int tile = (int)(blockIdx.x / (unsigned)a.groups), group = (int)(blockIdx.x % (unsigned)a.groups);
    const Piece p = a.ix.tiles[tile];
    if (!a.ix.good() || p.seq < 0) return;                       // (the same for every wave of the workgroup)
    int d = (group * CW + (GROUPS > 1 ? 0 : wave)) * 64 + lane;
    const bool on = d < a.D;
    if (!on) d = a.D - 1;                                        // lanes without a channel: another's inputs, no gradient
    float a2[kStates], g[kStates], dA[kStates];
    load_row(a2, a.A + (int64_t)d * a.N + n0, n0, a.N);
    const float bias = a.bias ? a.bias[d] : 0.f, skip = a.Dv ? a.Dv[d] : 0.f;
    const int64_t at = ((int64_t)tile * a.N + n0) * a.D + d;
    const bool sp = a.softplus != 0;
    float dskip = 0.f, dbias = 0.f;
#pragma unroll
    for (int n = 0; n < kStates; ++n) {
        a2[n] *= kLog2e;
        dA[n] = 0.f;
        g[n] = on && !(p.bits & 2) && n0 + n < a.N ? a.backs[at + (int64_t)n * a.D] : 0.f;
    }
    auto state_at_start = [&](int n) { return !(p.bits & 1) && n0 + n < a.N ? a.ends[at + (int64_t)n * a.D] : 0.f; };
    float* starts = s_starts + (int64_t)wave * start_slots(a.ix.tile) * kStates * 64 + lane;
    float* sb = s_b[wave];
    float* sc = s_c[wave];
    const int blocks = (p.count + kTok - 1) / kTok;

    // B (and C) of a block into this wave's LDS, [state][token]; a lane brings one token's states lane / 16 + 4 i
    auto stage_bc = [&](int first, int count, auto with_c) {
        const int t = lane & (kTok - 1);
        const int64_t row = first + min(t, count - 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = (lane >> 4) + 4 * i;
            const bool there = n0 + n < a.N;
            sb[n * kTok + t] = there ? Io<T>::ld(static_cast<const T*>(a.Bm) + row * a.b_stride + n0 + n) : 0.f;
            if constexpr (decltype(with_c)::value)
                sc[n * kTok + t] = there ? Io<T>::ld(static_cast<const T*>(a.Cm) + row * a.c_stride + n0 + n) : 0.f;
        }
    };
    // 16 tokens of one tensor, as stored; rows behind the piece are replaced by its last.  The row's address goes from token to token:
    // computed for each, the addresses of all tokens of all tensors would fill the scalar registers
    struct Tokens {
        T v[kTok];
    };
    auto load_tokens = [&](const void* base, int64_t stride, int first, int count) {
        const T* row = static_cast<const T*>(base) + first * stride;
        Tokens k;
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            k.v[t] = row[d];
            row += t + 1 < count ? stride : 0;
        }
        return k;
    };
    // step sizes and their products with u; 0 for tokens behind the piece
    auto load_steps = [&](int first, int count, float (&dl)[kTok], float (&dx)[kTok]) {
        const Tokens u = load_tokens(a.u, a.u_stride, first, count), delta = load_tokens(a.delta, a.d_stride, first, count);
#pragma unroll
        for (int t = 0; t < kTok; ++t) dl[t] = Io<T>::ld(&delta.v[t]) + bias;
        if (sp) corey_scan::softplus_all<kTok>(dl);
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            dl[t] = t < count ? dl[t] : 0.f;
            dx[t] = t < count ? dl[t] * Io<T>::ld(&u.v[t]) : 0.f;
        }
    };

    // forward over all blocks but the last: the states that blocks 1, 2, ... begin with
    if (blocks > 1) {
        float h[kStates];
#pragma unroll
        for (int n = 0; n < kStates; ++n) h[n] = state_at_start(n);
        for (int b = 0; b + 1 < blocks; ++b) {
            float dl[kTok], dx[kTok];
            lds_in_order();
            stage_bc(p.first + b * kTok, kTok, std::false_type());
            load_steps(p.first + b * kTok, kTok, dl, dx);
            lds_in_order();
#pragma unroll
            for (int n = 0; n < kStates; ++n) {
                float e[kTok];
#pragma unroll
                for (int t = 0; t < kTok; ++t) e[t] = dl[t] * a2[n];
                exp2_burst<kTok>(e);
                const Words<kTok> bv = words<kTok>(sb + n * kTok);
#pragma unroll
                for (int t = 0; t < kTok; ++t) h[n] = fmaf(e[t], h[n], dx[t] * bv.v[t]);
                starts[(b * kStates + n) * 64] = h[n];
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }

    for (int b = blocks - 1; b >= 0; --b) {
        const int first = p.first + b * kTok, count = min(kTok, p.count - b * kTok);
        float dl[kTok], dx[kTok], ds[kTok], gb[kTok], gk[kTok], out[kTok];
        lds_in_order();
        if (b == 0) {                                            // the first block's states, where block 1's were
#pragma unroll
            for (int n = 0; n < kStates; ++n) starts[n * 64] = state_at_start(n);
        }
        stage_bc(first, count, std::true_type());
        load_steps(first, count, dl, dx);
        {
            const Tokens dy = load_tokens(a.dy, a.dy_stride, first, count);
            Tokens z;
            if constexpr (GATED) z = load_tokens(a.z, a.z_stride, first, count);
#pragma unroll
            for (int t = 0; t < kTok; ++t) {
                ds[t] = Io<T>::ld(&dy.v[t]);
                if constexpr (GATED) ds[t] *= silu(Io<T>::ld(&z.v[t]));
                ds[t] = on && t < count ? ds[t] : 0.f;
                gb[t] = gk[t] = out[t] = 0.f;
            }
        }
        lds_in_order();
        const float* begin = starts + max(b - 1, 0) * kStates * 64;
#pragma unroll
        for (int n = 0; n < kStates; ++n) {
            float h = begin[n * 64];
            float e[kTok], w[kTok], v[kTok];
#pragma unroll
            for (int t = 0; t < kTok; ++t) e[t] = dl[t] * a2[n];
            exp2_burst<kTok>(e);
#pragma unroll
            for (int q = 0; q < kTok; q += 4) {                  // (B and C four tokens at a time, and again on the way back)
                const Words<4> bv = words<4>(sb + n * kTok + q), cv = words<4>(sc + n * kTok + q);
#pragma unroll
                for (int t = q; t < q + 4; ++t) {
                    w[t] = e[t] * h;                             // a h_{t-1}
                    h = fmaf(dx[t], bv.v[t - q], w[t]);
                    out[t] = fmaf(cv.v[t - q], h, out[t]);
                    v[t] = ds[t] * h;
                }
            }
            const float sum_c = fold16(v, lane);
            float gn = g[n], an = dA[n];
            asm volatile("" ::: "memory");
#pragma unroll
            for (int q = kTok - 4; q >= 0; q -= 4) {
                const Words<4> bv = words<4>(sb + n * kTok + q), cv = words<4>(sc + n * kTok + q);
#pragma unroll
                for (int t = q + 3; t >= q; --t) {
                    gn = fmaf(ds[t], cv.v[t - q], gn);
                    gb[t] = fmaf(gn, bv.v[t - q], gb[t]);
                    const float through = gn * w[t];
                    gk[t] = fmaf(a2[n], through, gk[t]);
                    an = fmaf(dl[t], through, an);
                    v[t] = gn * dx[t];
                    gn *= e[t];
                }
            }
            const float sum_b = fold16(v, lane);
            s_fold[wave][n * kFold + 2 * (lane >> 2) + (lane & 1)] = (lane & 1) ? sum_c : sum_b;      // (two lanes each, the same value)
            // a state's share of the sums is added here: the compiler would rather keep all states' values and add them up at the end
#pragma unroll
            for (int t = 0; t < kTok; ++t) asm volatile("" : "+v"(gb[t]), "+v"(gk[t]), "+v"(out[t])::"memory");
            asm volatile("" : "+v"(gn), "+v"(an));
            g[n] = gn;
            dA[n] = an;
            __builtin_amdgcn_sched_barrier(0);
        }
        // dB and dC of the block, over the workgroup's channels
        if constexpr (GROUPS == 1) {
            __syncthreads();
            for (int i = (int)threadIdx.x; i < kTok * 2 * kStates; i += 64 * WAVES) {
                const int t = i >> 5, bc = (i >> 4) & 1, n = i & (kStates - 1);
                if (t < count && n < a.N) {
                    float sum = 0.f;
#pragma unroll
                    for (int k = 0; k < WAVES; ++k) sum += s_fold[k][n * kFold + 2 * t + bc];
                    a.part_bc[((int64_t)group * a.ix.T + first + t) * 2 * a.N + bc * a.N + n] = sum;
                }
            }
            __syncthreads();
        } else {
            lds_in_order();
            for (int i = lane; i < kTok * 2 * kStates; i += 64) {
                const int t = i >> 5, bc = (i >> 4) & 1, n = i & (kStates - 1);
                if (t < count && n0 + n < a.N)
                    a.part_bc[((int64_t)group * a.ix.T + first + t) * 2 * a.N + bc * a.N + n0 + n] = s_fold[wave][n * kFold + 2 * t + bc];
            }
            // the sums over the waves' states; wave 0 finishes
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
            for (int k = 1; k < GROUPS; ++k) {
#pragma unroll
                for (int t = 0; t < kTok; ++t) {
                    gb[t] += s_part[k - 1][t * 64 + lane];
                    gk[t] += s_part[k - 1][(kTok + t) * 64 + lane];
                    out[t] += s_part[k - 1][(2 * kTok + t) * 64 + lane];
                }
            }
        }
        // what only the end needs is read again (from the cache): kept, it would take the registers of a state's work
        const Tokens ku = load_tokens(a.u, a.u_stride, first, count), kd = load_tokens(a.delta, a.d_stride, first, count);
        Tokens kz, ky;
        if constexpr (GATED) {
            kz = load_tokens(a.z, a.z_stride, first, count);
            ky = load_tokens(a.dy, a.dy_stride, first, count);
        }
        T* du_row = static_cast<T*>(a.du) + first * a.du_stride;
        T* dd_row = static_cast<T*>(a.ddelta) + first * a.dd_stride;
        T* dz_row = GATED ? static_cast<T*>(a.dz) + first * a.dz_stride : nullptr;
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            const float u = Io<T>::ld(&ku.v[t]);
            float ddl = fmaf(u, gb[t], gk[t] * kLn2);
            if (sp) ddl *= __builtin_amdgcn_rcpf(1.f + fast_exp2(-(Io<T>::ld(&kd.v[t]) + bias) * kLog2e));
            const float du = fmaf(skip, ds[t], dl[t] * gb[t]);
            float dz = 0.f;
            if constexpr (GATED) {
                const float z = Io<T>::ld(&kz.v[t]), sig = __builtin_amdgcn_rcpf(1.f + fast_exp2(-z * kLog2e));
                dz = Io<T>::ld(&ky.v[t]) * fmaf(skip, u, out[t]) * (sig * fmaf(z, 1.f - sig, 1.f));
            }
            if (on && t < count) {
                Io<T>::st(du_row + d, du);
                Io<T>::st(dd_row + d, ddl);
                if constexpr (GATED) Io<T>::st(dz_row + d, dz);
            }
            dskip = t < count ? fmaf(ds[t], u, dskip) : dskip;
            dbias = t < count ? dbias + ddl : dbias;
            du_row += a.du_stride;
            dd_row += a.dd_stride;
            if constexpr (GATED) dz_row += a.dz_stride;
        }
    }
    if (!on) return;
    float* part = a.part_a + (int64_t)tile * (a.N + 2) * a.D + d;
#pragma unroll
    for (int n = 0; n < kStates; ++n)
        if (n0 + n < a.N) part[(int64_t)(n0 + n) * a.D] = dA[n];
    if (n0 == 0) {
        part[(int64_t)a.N * a.D] = dskip;
        part[(int64_t)(a.N + 1) * a.D] = dbias;
    }
}

// dB and dC: the workgroups' sums, one value a lane.
template <typename T> __global__ __launch_bounds__(256) void k_packed_bwd_bc(PackedScanArgs a)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, wide = 2 * a.N;
    if (!a.ix.good() || i >= a.ix.head[4] * wide) return;
    const int64_t t = i / wide;
    const int j = (int)(i - t * wide);
    float sum = 0.f;
    for (int g = 0; g < a.groups; ++g) sum += a.part_bc[(int64_t)g * a.ix.T * wide + i];
    if (j < a.N) Io<T>::st(static_cast<T*>(a.dB) + t * a.db_stride + j, sum);
    else Io<T>::st(static_cast<T*>(a.dC) + t * a.dc_stride + (j - a.N), sum);
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
    int64_t ends, backs, sums, part_bc, part_a, all;
};
Space space(const Layout& l, int64_t T, int32_t tile, int64_t D, int64_t N)
{
    const int64_t tiles = T > tile ? l.max_tiles : 0;            // (carried only where a sequence can have a second tile)
    const int64_t groups = N <= kStates ? (D + 255) / 256 : (D + 63) / 64;
    Space s;
    s.ends = 0;
    s.backs = s.ends + tiles * N * D;
    s.sums = s.backs + tiles * N * D;
    s.part_bc = s.sums + tiles * D;
    s.part_a = s.part_bc + groups * T * 2 * N;
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
    a.ends = ws + w.ends; a.backs = ws + w.backs; a.sums = ws + w.sums; a.part_bc = ws + w.part_bc; a.part_a = ws + w.part_a;
    a.D = (int32_t)D; a.N = (int32_t)N;
    a.softplus = delta_softplus ? 1 : 0;
    a.tiles = (int32_t)l.max_tiles;
    const int64_t pairs = (D + 127) / 128, columns = (D * N + 255) / 256, groups = N <= kStates ? (D + 255) / 256 : (D + 63) / 64;
    const int64_t bc = (pack->T * 2 * N + 255) / 256;
    if (l.max_tiles * groups > INT32_MAX || l.max_tiles * pairs > INT32_MAX || 2 * columns * (l.max_longs + 1) > INT32_MAX || bc > INT32_MAX)
        return fail(COREY_ESHAPE, "%s: T * D is too large", who);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    hipError_t attr = hipSuccess;
    by_type(dt, [&](auto t) {
        using T = decltype(t);
        by_groups(N, [&](auto gr) {
            constexpr int G = decltype(gr)::value;
            auto go = [&](auto gate) {
                constexpr bool Z = decltype(gate)::value;
                const size_t lds = (size_t)back_waves<G>() * (size_t)start_slots(pack->tile) * kStates * 64 * 4;
                // (what the longest tile takes, whatever this call's: another thread's call may be between this line and its launch)
                constexpr int most = back_waves<G>() * start_slots(G == 8 ? 32 : kMaxBackTile) * kStates * 64 * 4;
                attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_packed_bwd<T, Z, G>), hipFuncAttributeMaxDynamicSharedMemorySize, most);
                if (attr != hipSuccess) return;
                if (pack->T > pack->tile) {
                    a.groups = (int32_t)pairs;
                    const unsigned grid = (unsigned)(l.max_tiles * pairs);
                    if (D % 2 == 0) k_packed_bwd_ends<T, true, Z, G><<<grid, 64 * G, 0, stream>>>(a);
                    else k_packed_bwd_ends<T, false, Z, G><<<grid, 64 * G, 0, stream>>>(a);
                    k_packed_bwd_chain<<<(unsigned)(2 * columns * l.max_longs), 256, 0, stream>>>(a, (int)columns);
                }
                a.groups = (int32_t)groups;
                k_packed_bwd<T, Z, G><<<(unsigned)(l.max_tiles * groups), 64 * back_waves<G>(), lds, stream>>>(a);
            };
            if (z) go(std::true_type());
            else go(std::false_type());
        });
        if (attr == hipSuccess) k_packed_bwd_bc<T><<<(unsigned)bc, 256, 0, stream>>>(a);
    });
    if (attr != hipSuccess) return corey::hip_fail(attr, "corey_scan_packed_bwd: LDS");
    k_packed_bwd_a<<<(unsigned)(((N + 2) * D + 63) / 64), 256, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? corey::hip_fail(e, "corey_scan_packed_bwd launch") : COREY_OK;
}
