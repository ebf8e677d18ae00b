// corey_conv_packed and corey_conv_packed_bwd: the causal depthwise convolution with SiLU on packed batches, and its gradients.
//
//     v[t] = bias + sum_k w[k] x[t - (W-1) + k] inside the sequence (before its first token: the slot's state, else 0)
//     u[t] = v sigmoid(v)
//
// Memory bound: 2 values per token and channel forward, 3 backward.  A lane holds V neighbouring channels (four where D allows) and a
// wave a piece of at most 16 tokens, whose rows it requests eight together; the W-1 rows before the piece come from the cache (the
// neighbouring piece is the same workgroup's).  16384 tokens of 5120 bf16 channels (337 MB), us: one piece a wave 74, runs of 2, 4, 8, 16
// pieces, which keep the taps, 78, 83, 83, 101; eight channels a lane as long as four.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "corey_packed.h"
#include "corey_scan_impl.h"

namespace {

using namespace corey_packed;
using corey_scan::fast_exp2;
using corey_scan::Io;
using corey_scan::kLog2e;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

template <typename T, int V> struct Vec {       // V channels of a token, as stored
    T v[V];
};
template <typename T, int V> __device__ __forceinline__ Vec<T, V> load(const T* p)
{
    Vec<T, V> r;
    __builtin_memcpy(&r, p, sizeof(r));
    return r;
}
template <typename T, int V> __device__ __forceinline__ void store(T* p, const float (&f)[V])
{
    if constexpr (sizeof(T) == 2) {                              // rounded two at a time
        constexpr int P = (V + 1) / 2;
        uint32_t w[P];
#pragma unroll
        for (int i = 0; i < P; ++i) w[i] = Io<T>::pack2(f[2 * i], f[2 * i + 1 < V ? 2 * i + 1 : 2 * i]);
        __builtin_memcpy(p, w, V * sizeof(T));
    } else {
        __builtin_memcpy(p, f, sizeof(f));
    }
}

__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + fast_exp2(-v * kLog2e)); }

struct ConvArgs {
    Index ix;
    const void *x, *state;                      // state: [n_slots, D, W-1]
    const float *weight, *bias;
    const int32_t *slots, *slots_out;
    void *u, *state_out;                        // state_out: the same pool
    int64_t x_stride, u_stride, n_slots;
    int32_t D, groups, pieces;                  // groups: of 64 V channels
    // backward
    const void* du;
    void* dx;
    int64_t du_stride, dx_stride;
    float* parts;                               // [runs, W + 1, D] sums of a run of pieces
    int32_t run, runs;
};

template <typename T, int V, int W> __device__ __forceinline__ void load_taps(const ConvArgs& a, int d, float (&w)[W][V], float (&b)[V])
{
    float rows[V][W];                           // [D, W]: a lane's channels are one stretch
    __builtin_memcpy(rows, a.weight + (int64_t)d * W, sizeof(rows));
#pragma unroll
    for (int i = 0; i < V; ++i) {
        b[i] = a.bias ? a.bias[d + i] : 0.f;
#pragma unroll
        for (int k = 0; k < W; ++k) w[k][i] = rows[i][k];
    }
}

template <typename T, int V, int W>
__global__ __launch_bounds__(kThreads) void k_conv_packed(ConvArgs a)
{
    const int group = (int)(blockIdx.x % (unsigned)a.groups);
    const int64_t at = (int64_t)(blockIdx.x / (unsigned)a.groups) * kWaves + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (at >= a.pieces || !a.ix.good()) return;
    const Piece p = a.ix.blocks[at];
    if (p.seq < 0) return;
    const int d = (group * 64 + ((int)threadIdx.x & 63)) * V;
    if (d >= a.D) return;
    constexpr int H = W - 1;
    const T* x = static_cast<const T*>(a.x) + d;
    T* u = static_cast<T*>(a.u) + d;
    const int64_t xs = a.x_stride;
    float w[W][V], b[V];
    load_taps<T, V, W>(a, d, w, b);
    float past[H > 0 ? H : 1][V] = {};          // the inputs before the next token, oldest first
    const bool first = (p.bits & 1) != 0;
    // groups of tokens: the rows of a group are requested together
    auto tokens = [&](int t0, auto count) {
        constexpr int C = decltype(count)::value;
        Vec<T, V> r[C];
#pragma unroll
        for (int t = 0; t < C; ++t) r[t] = load<T, V>(x + (int64_t)(p.first + t0 + t) * xs);
#pragma unroll
        for (int t = 0; t < C; ++t) {
            float now[V], out[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                now[i] = Io<T>::ld(&r[t].v[i]);
                float s = b[i];
#pragma unroll
                for (int k = 0; k < H; ++k) s = fmaf(w[k][i], past[k][i], s);
                s = fmaf(w[H][i], now[i], s);
                out[i] = s * sigmoid(s);
            }
            store<T, V>(u + (int64_t)(p.first + t0 + t) * a.u_stride, out);
#pragma unroll
            for (int i = 0; i < V; ++i) {
#pragma unroll
                for (int k = 0; k + 1 < H; ++k) past[k][i] = past[k + 1][i];
                if constexpr (H > 0) past[H - 1][i] = now[i];
            }
        }
    };
    T old[V][H > 0 ? H : 1] = {};
    if constexpr (H > 0) {
        if (first) {
            const int64_t from = slot_of(a.slots, p.seq, a.n_slots);
            if (from >= 0) __builtin_memcpy(old, static_cast<const T*>(a.state) + (from * a.D + d) * H, sizeof(old));
#pragma unroll
            for (int j = 0; j < H; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) past[j][i] = Io<T>::ld(&old[i][j]);
        } else {                                // (pieces before the last have 16 tokens: all of these are the sequence's)
#pragma unroll
            for (int j = 0; j < H; ++j) {
                const Vec<T, V> r = load<T, V>(x + (int64_t)(p.first - H + j) * xs);
#pragma unroll
                for (int i = 0; i < V; ++i) past[j][i] = Io<T>::ld(&r.v[i]);
            }
        }
    }
    if (p.count == kBlock) {
#pragma unroll 1
        for (int t = 0; t < kBlock; t += kBlock / 2) tokens(t, std::integral_constant<int, kBlock / 2>());
    } else {
        int t = 0;
        for (; t + 4 <= p.count; t += 4) tokens(t, std::integral_constant<int, 4>());
        for (; t < p.count; ++t) tokens(t, std::integral_constant<int, 1>());
    }
    // The state moves on: the last W-1 of (old state, inputs).  The wave that has read the old state writes the new one, so a
    // slot that is read and written by one sequence is in no race.
    if constexpr (H > 0) {
        const int64_t to = first ? slot_of(a.slots_out, p.seq, a.n_slots) : -1;
        if (to < 0) return;
        const int begin = p.first, len = a.ix.starts[p.seq + 1] - begin;
        T now[V][H];
#pragma unroll
        for (int j = 0; j < H; ++j) {
            const int t = len - H + j;      // before the first token: the old state's
            if (t >= 0) {
                const Vec<T, V> r = load<T, V>(x + (int64_t)(begin + t) * xs);
#pragma unroll
                for (int i = 0; i < V; ++i) now[i][j] = r.v[i];
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    now[i][j] = T(0);
#pragma unroll
                    for (int o = 0; o < H; ++o) now[i][j] = o == H + t ? old[i][o] : now[i][j];
                }
            }
        }
        __builtin_memcpy(static_cast<T*>(a.state_out) + (to * a.D + d) * H, now, sizeof(now));
    }
}

// Gradients.  With dv[t] = du[t] silu'(v[t]):  dx[t] = sum_k w[k] dv[t + (W-1) - k] (0 behind the sequence's end),
// dw[k] = sum_t dv[t] x[t - (W-1) + k], dbias = sum_t dv[t].  v is formed again.  A wave walks a run of pieces and keeps the last W
// dv and its sums of dw and dbias in registers; dx lies W-1 tokens behind, and where the run ends inside a sequence the next W-1
// tokens are looked at for it.  A second kernel adds up the runs, always in the same order.
template <typename T, int V, int W>
__global__ __launch_bounds__(kThreads) void k_conv_packed_bwd(ConvArgs a)
{
    const int group = (int)(blockIdx.x % (unsigned)a.groups);
    const int64_t run = (int64_t)(blockIdx.x / (unsigned)a.groups) * kWaves + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (run >= a.runs || !a.ix.good()) return;
    const int d = (group * 64 + ((int)threadIdx.x & 63)) * V;
    if (d >= a.D) return;
    constexpr int H = W - 1;
    const T* x = static_cast<const T*>(a.x) + d;
    const T* du = static_cast<const T*>(a.du) + d;
    T* dx = static_cast<T*>(a.dx) + d;
    float w[W][V], b[V], dw[W][V] = {}, db[V] = {};
    load_taps<T, V, W>(a, d, w, b);
    float past[H > 0 ? H : 1][V] = {}, dv[W][V] = {};            // the inputs before the next token; dv of the last W, oldest first
    int behind = 0;                             // tokens (at most W-1) whose dx is still to come
    // dv of one more token joins, and the dx that it completes (of the token W-1 rows before `row`) is stored
    const auto join = [&](int64_t row, const float (&g)[V]) {
        float out[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
#pragma unroll
            for (int k = 0; k < H; ++k) dv[k][i] = dv[k + 1][i];
            dv[H][i] = g[i];
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < W; ++k) sum = fmaf(w[k][i], dv[H - k][i], sum);
            out[i] = sum;
        }
        if (behind == H) store<T, V>(dx + (row - H) * a.dx_stride, out);
        else ++behind;
    };
    const auto tokens = [&](int64_t row, auto count, auto mine) {      // (mine: they count for dw and dbias)
        constexpr int C = decltype(count)::value;
        Vec<T, V> rx[C], rg[C];
#pragma unroll
        for (int t = 0; t < C; ++t) {
            rx[t] = load<T, V>(x + (row + t) * a.x_stride);
            rg[t] = load<T, V>(du + (row + t) * a.du_stride);
        }
#pragma unroll
        for (int t = 0; t < C; ++t) {
            float g[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float now = Io<T>::ld(&rx[t].v[i]);
                float s = b[i];
#pragma unroll
                for (int k = 0; k < H; ++k) s = fmaf(w[k][i], past[k][i], s);
                s = fmaf(w[H][i], now, s);
                const float sig = sigmoid(s);
                g[i] = Io<T>::ld(&rg[t].v[i]) * (sig * fmaf(s, 1.f - sig, 1.f));
                if constexpr (decltype(mine)::value) {
#pragma unroll
                    for (int k = 0; k < H; ++k) dw[k][i] = fmaf(g[i], past[k][i], dw[k][i]);
                    dw[H][i] = fmaf(g[i], now, dw[H][i]);
                    db[i] += g[i];
                }
#pragma unroll
                for (int k = 0; k + 1 < H; ++k) past[k][i] = past[k + 1][i];
                if constexpr (H > 0) past[H - 1][i] = now;
            }
            join(row + t, g);
        }
    };
    using One = std::integral_constant<int, 1>;
    const int64_t stop = min((int64_t)a.pieces, (run + 1) * a.run);
    for (int64_t at = run * a.run; at < stop; ++at) {
        const Piece p = a.ix.blocks[at];
        if (p.seq < 0) break;                   // the used pieces come first
        if ((p.bits & 1) || at == run * a.run) {
            behind = 0;
#pragma unroll
            for (int j = 0; j < H; ++j) {
                if (p.bits & 1) {
#pragma unroll
                    for (int i = 0; i < V; ++i) past[j][i] = 0.f;
                } else {
                    const Vec<T, V> r = load<T, V>(x + (int64_t)(p.first - H + j) * a.x_stride);
#pragma unroll
                    for (int i = 0; i < V; ++i) past[j][i] = Io<T>::ld(&r.v[i]);
                }
            }
        }
        if (p.count == kBlock) {
#pragma unroll 1
            for (int t = 0; t < kBlock; t += kBlock / 2) tokens((int64_t)p.first + t, std::integral_constant<int, kBlock / 2>(), std::true_type());
        } else {
            for (int t = 0; t < p.count; ++t) tokens((int64_t)p.first + t, One(), std::true_type());
        }
        if constexpr (H > 0) {
            if (!(p.bits & 2) && at + 1 < stop) continue;
            // the sequence or the run ends: what follows completes the dx still to come (nothing follows a sequence)
            const int64_t row = (int64_t)p.first + p.count;
            const int follow = (int)min((int64_t)H, (int64_t)a.ix.starts[p.seq + 1] - row);
            const float none[V] = {};
            const int due = behind;
            // (a sequence shorter than W-1: its first dx is complete only when as many have joined)
            for (int j = 0, left = due; left > 0; ++j) {
                const bool out = behind == H;
                if (j < follow) tokens(row + j, One(), std::false_type());
                else join(row + j, none);
                left -= out ? 1 : 0;
            }
        }
    }
#pragma unroll
    for (int k = 0; k < W + 1; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) a.parts[((int64_t)run * (W + 1) + k) * a.D + d + i] = k < W ? dw[k < W ? k : 0][i] : db[i];
}

// Sums over the runs, [runs, W + 1, D] -> dweight [D, W] and dbias [D].  A workgroup takes 64 columns; its waves the runs in turn.
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(64 * kSumWaves) void k_conv_packed_sum(ConvArgs a, int W, float* dweight, float* dbias)
{
    __shared__ float part[kSumWaves][64];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int64_t n = (int64_t)(W + 1) * a.D, col = (int64_t)blockIdx.x * 64 + lane;
    float s[4] = {};
    if (col < n && a.ix.good()) {
        int r = wave;
        for (; r + 3 * kSumWaves < a.runs; r += 4 * kSumWaves) {
#pragma unroll
            for (int q = 0; q < 4; ++q) s[q] += a.parts[(r + q * kSumWaves) * n + col];
        }
        for (; r < a.runs; r += kSumWaves) s[0] += a.parts[r * n + col];
    }
    part[wave][lane] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (wave != 0 || col >= n || !a.ix.good()) return;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kSumWaves; ++w) sum += part[w][lane];
    const int k = (int)(col / a.D), d = (int)(col % a.D);
    if (k < W) dweight[(int64_t)d * W + k] = sum;
    else if (dbias) dbias[d] = sum;
}

// Channels of a lane: four, or as many as D is whole numbers of (a lane's channels are all there or none is).
template <typename F> void by_width(int64_t D, F&& f)
{
    if (D % 4 == 0) return f(std::integral_constant<int, 4>());
    if (D % 2 == 0) return f(std::integral_constant<int, 2>());
    return f(std::integral_constant<int, 1>());
}
int64_t groups_of(int64_t D)                    // of 64 lanes' channels
{
    int64_t wide = 0;
    by_width(D, [&](auto v) { wide = 64 * decltype(v)::value; });
    return (D + wide - 1) / wide;
}
template <typename F> void by_taps(int W, F&& f)
{
    if (W == 1) f(std::integral_constant<int, 1>());
    else if (W == 2) f(std::integral_constant<int, 2>());
    else if (W == 3) f(std::integral_constant<int, 3>());
    else f(std::integral_constant<int, 4>());
}

// Runs of pieces the backward pass is cut into: as many waves as the GPU runs at once, three a SIMD by their registers.  16384 tokens of
// 5120 bf16 channels, us: one wave a SIMD 177, two 129, three 120, four 136, eight 128.
constexpr int64_t kWavesAtOnce = 3 * 4 * 256;
int64_t runs_of(int64_t pieces, int64_t groups, int32_t* run)
{
    const int64_t want = std::max<int64_t>(1, kWavesAtOnce / groups);
    *run = (int32_t)((pieces + want - 1) / want);
    return (pieces + *run - 1) / *run;
}

int check_common(const char* who, const corey_pack* pack, Index* ix, const void* x, const float* weight, corey_dtype dt, int64_t D, int32_t W)
{
    using corey::fail;
    if (!x || !weight) return fail(COREY_ENULL, "%s: x and weight are required", who);
    if (!good_dtype(dt)) return fail(COREY_EINVAL, "%s: unknown dtype %d", who, (int)dt);
    if (W < 1 || W > COREY_MAX_CONV) return fail(COREY_EINVAL, "%s: 1 <= W <= %d required", who, COREY_MAX_CONV);
    if (D < 1 || D > COREY_PACK_MAX_CHANNELS) return fail(COREY_ESHAPE, "%s: 1 <= D <= %d required", who, COREY_PACK_MAX_CHANNELS);
    return index_of(who, pack, ix);
}

}  // namespace

extern "C" int corey_conv_packed(const void* x, int64_t x_stride, const float* weight, const float* bias, void* state, int64_t n_slots,
                                 const int32_t* slots, const int32_t* slots_out, const corey_pack* pack, void* u, int64_t u_stride,
                                 corey_dtype dt, int64_t D, int32_t W, void* hip_stream)
{
    using corey::fail;
    const char* who = "corey_conv_packed";
    ConvArgs a = {};
    if (int e = check_common(who, pack, &a.ix, x, weight, dt, D, W)) return e;
    if (!u) return fail(COREY_ENULL, "%s: u is required", who);
    if (u == x) return fail(COREY_EINVAL, "%s: u may not be x", who);
    if (!good_stride(x_stride, D) || !good_stride(u_stride, D)) return fail(COREY_ESHAPE, "%s: rows must be at least D apart", who);
    if (W > 1 && (slots || slots_out) && (!state || n_slots < 1)) return fail(COREY_ENULL, "%s: slots need a pool of states", who);
    const Layout l = layout(pack->S, pack->T, pack->tile);
    a.x = x;
    a.state = state;
    a.state_out = state;
    a.weight = weight;
    a.bias = bias;
    a.slots = slots;
    a.slots_out = slots_out ? slots_out : slots;
    a.n_slots = n_slots;
    a.u = u;
    a.x_stride = x_stride;
    a.u_stride = u_stride;
    a.D = (int32_t)D;
    a.pieces = (int32_t)l.max_blocks;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    bool fits = true;
    by_type(dt, [&](auto t) {
        using T = decltype(t);
        by_width(D, [&](auto v) {
            constexpr int V = decltype(v)::value;
            a.groups = (int32_t)groups_of(D);
            const int64_t grid = (l.max_blocks + kWaves - 1) / kWaves * a.groups;
            fits = good_grid(grid, kThreads);
            if (!fits) return;
            by_taps(W, [&](auto w) { k_conv_packed<T, V, decltype(w)::value><<<(unsigned)grid, kThreads, 0, stream>>>(a); });
        });
    });
    if (!fits) return fail(COREY_ESHAPE, "%s: T * D is too large", who);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? corey::hip_fail(e, "corey_conv_packed launch") : COREY_OK;
}

extern "C" size_t corey_conv_packed_bwd_workspace(const corey_pack* pack, int64_t D, int32_t W)
{
    Index ix;
    if (W < 1 || W > COREY_MAX_CONV || D < 1 || D > COREY_PACK_MAX_CHANNELS || index_of("corey_conv_packed_bwd_workspace", pack, &ix)) return 0;
    int32_t run;
    return (size_t)(runs_of(layout(pack->S, pack->T, pack->tile).max_blocks, groups_of(D), &run) * (W + 1) * D) * 4;
}

extern "C" int corey_conv_packed_bwd(const void* x, int64_t x_stride, const float* weight, const float* bias, const void* du,
                                     int64_t du_stride, const corey_pack* pack, void* dx, int64_t dx_stride, float* dweight, float* dbias,
                                     corey_dtype dt, int64_t D, int32_t W, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    using corey::fail;
    const char* who = "corey_conv_packed_bwd";
    ConvArgs a = {};
    if (int e = check_common(who, pack, &a.ix, x, weight, dt, D, W)) return e;
    if (!du || !dx || !dweight) return fail(COREY_ENULL, "%s: du, dx and dweight are required", who);
    if (dx == x || dx == du) return fail(COREY_EINVAL, "%s: dx may not be an input", who);
    if (!good_stride(x_stride, D) || !good_stride(du_stride, D) || !good_stride(dx_stride, D))
        return fail(COREY_ESHAPE, "%s: rows must be at least D apart", who);
    if (!workspace || workspace_bytes < corey_conv_packed_bwd_workspace(pack, D, W) || reinterpret_cast<uintptr_t>(workspace) % 4 != 0)
        return fail(COREY_EWORKSPACE, "%s: workspace missing, misaligned or smaller than corey_conv_packed_bwd_workspace()", who);
    const Layout l = layout(pack->S, pack->T, pack->tile);
    a.x = x;
    a.weight = weight;
    a.bias = bias;
    a.du = du;
    a.dx = dx;
    a.x_stride = x_stride;
    a.du_stride = du_stride;
    a.dx_stride = dx_stride;
    a.D = (int32_t)D;
    a.pieces = (int32_t)l.max_blocks;
    a.parts = static_cast<float*>(workspace);
    a.groups = (int32_t)groups_of(D);
    a.runs = (int32_t)runs_of(l.max_blocks, a.groups, &a.run);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const unsigned grid = (unsigned)((a.runs + kWaves - 1) / kWaves * a.groups);
    by_type(dt, [&](auto t) {
        by_width(D, [&](auto v) {
            by_taps(W, [&](auto w) { k_conv_packed_bwd<decltype(t), decltype(v)::value, decltype(w)::value><<<grid, kThreads, 0, stream>>>(a); });
        });
    });
    k_conv_packed_sum<<<(unsigned)(((W + 1) * D + 63) / 64), 64 * kSumWaves, 0, stream>>>(a, W, dweight, dbias);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? corey::hip_fail(e, "corey_conv_packed_bwd launch") : COREY_OK;
}
