// corey_conv_packed and corey_conv_packed_bwd: the causal depthwise convolution with SiLU on packed batches, and its gradients.
//
//     v[t] = bias + sum_k w[k] x[t - (W-1) + k] inside the sequence (before its first token: the slot's state, else 0)
//     u[t] = v sigmoid(v)
//
// Memory bound: 2 values per token and channel forward, 3 backward.  A lane holds V neighbouring channels (16 bytes of them where
// D allows) and a wave one piece of at most 16 tokens, whose rows it requests all at once, the W-1 rows before it again (they come
// from the cache, the neighbouring piece is the same workgroup's).
#include <hip/hip_runtime.h>

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
    Vec<T, V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) Io<T>::st(&r.v[i], f[i]);
    __builtin_memcpy(p, &r, sizeof(r));
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
    const int64_t xs = a.x_stride;
    float w[W][V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        b[i] = a.bias ? a.bias[d + i] : 0.f;
#pragma unroll
        for (int k = 0; k < W; ++k) w[k][i] = a.weight[(int64_t)(d + i) * W + k];
    }
    float past[H > 0 ? H : 1][V] = {};          // the inputs before the piece, oldest first
    const bool first = (p.bits & 1) != 0;
    const int64_t from = first ? slot_of(a.slots, p.seq, a.n_slots) : -1;
    T old[V][H > 0 ? H : 1] = {};
    if constexpr (H > 0) {
        if (!first) {                           // (pieces before the last have 16 tokens: all of these are the sequence's)
#pragma unroll
            for (int j = 0; j < H; ++j) {
                const Vec<T, V> r = load<T, V>(x + (p.first - H + j) * xs);
#pragma unroll
                for (int i = 0; i < V; ++i) past[j][i] = Io<T>::ld(&r.v[i]);
            }
        } else if (from >= 0) {
            __builtin_memcpy(old, static_cast<const T*>(a.state) + (from * a.D + d) * H, sizeof(old));
#pragma unroll
            for (int j = 0; j < H; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) past[j][i] = Io<T>::ld(&old[i][j]);
        }
    }
    T* u = static_cast<T*>(a.u) + d;
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
    if (p.count == kBlock) {
        tokens(0, std::integral_constant<int, kBlock>());
    } else {
        int t = 0;
        for (; t + 4 <= p.count; t += 4) tokens(t, std::integral_constant<int, 4>());
        for (; t < p.count; ++t) tokens(t, std::integral_constant<int, 1>());
    }
    // The state moves on: the last W-1 of (old state, inputs).  The wave that has read the old state writes the new one, so a
    // slot that is read and written by one sequence is in no race.
    if constexpr (H > 0) {
        if (!first) return;
        const int64_t to = slot_of(a.slots_out, p.seq, a.n_slots);
        if (to < 0) return;
        const int begin = p.first, len = a.ix.starts[p.seq + 1] - begin;
        T now[V][H];
#pragma unroll
        for (int j = 0; j < H; ++j) {
            const int t = len - H + j;          // before the first token: the old state's
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
// dw[k] = sum_t dv[t] x[t - (W-1) + k], dbias = sum_t dv[t].  v is formed again.  A wave walks a run of pieces and keeps its sums
// of dw and dbias in registers; a second kernel adds up the runs, always in the same order.
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
#pragma unroll
    for (int i = 0; i < V; ++i) {
        b[i] = a.bias ? a.bias[d + i] : 0.f;
#pragma unroll
        for (int k = 0; k < W; ++k) w[k][i] = a.weight[(int64_t)(d + i) * W + k];
    }
    const int64_t stop = min((int64_t)a.pieces, (run + 1) * a.run);
    for (int64_t at = run * a.run; at < stop; ++at) {
        const Piece p = a.ix.blocks[at];
        if (p.seq < 0) break;                   // the used pieces come first
        const int end = a.ix.starts[p.seq + 1];
        const int ahead = min(H, end - (p.first + p.count));       // tokens behind the piece whose dv its dx needs
        float past[H > 0 ? H : 1][V] = {}, dv[W][V] = {};           // dv: of the last W tokens, oldest first
        if constexpr (H > 0) {
            if (!(p.bits & 1)) {
#pragma unroll
                for (int j = 0; j < H; ++j) {
                    const Vec<T, V> r = load<T, V>(x + (p.first - H + j) * a.x_stride);
#pragma unroll
                    for (int i = 0; i < V; ++i) past[j][i] = Io<T>::ld(&r.v[i]);
                }
            }
        }
        // token e of the piece (or behind it); dx of token e - H is ready then
        auto token = [&](int e, const Vec<T, V>& rx, const Vec<T, V>& rg, bool real, bool mine) {
            float out[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float now = Io<T>::ld(&rx.v[i]);
                float s = b[i];
#pragma unroll
                for (int k = 0; k < H; ++k) s = fmaf(w[k][i], past[k][i], s);
                s = fmaf(w[H][i], now, s);
                const float sig = sigmoid(s);
                const float g = real ? Io<T>::ld(&rg.v[i]) * (sig * fmaf(s, 1.f - sig, 1.f)) : 0.f;
#pragma unroll
                for (int k = 0; k < H; ++k) dv[k][i] = dv[k + 1][i];
                dv[H][i] = g;
                const float own = mine ? g : 0.f;
#pragma unroll
                for (int k = 0; k < H; ++k) dw[k][i] = fmaf(own, past[k][i], dw[k][i]);
                dw[H][i] = fmaf(own, now, dw[H][i]);
                db[i] += own;
                float sum = 0.f;
#pragma unroll
                for (int k = 0; k < W; ++k) sum = fmaf(w[k][i], dv[H - k][i], sum);
                out[i] = sum;
#pragma unroll
                for (int k = 0; k + 1 < H; ++k) past[k][i] = past[k + 1][i];
                if constexpr (H > 0) past[H - 1][i] = now;
            }
            if (e >= H) store<T, V>(dx + (int64_t)(p.first + e - H) * a.dx_stride, out);
        };
        auto tokens = [&](int e0, auto count) {
            constexpr int C = decltype(count)::value;
            Vec<T, V> rx[C], rg[C];
#pragma unroll
            for (int t = 0; t < C; ++t) {       // rows behind the sequence are replaced by its last
                const int64_t row = min((int64_t)p.first + e0 + t, (int64_t)end - 1);
                rx[t] = load<T, V>(x + row * a.x_stride);
                rg[t] = load<T, V>(du + row * a.du_stride);
            }
#pragma unroll
            for (int t = 0; t < C; ++t) {
                const int e = e0 + t;
                token(e, rx[t], rg[t], e < p.count + ahead, e < p.count);
            }
        };
        if (p.count == kBlock) {
            tokens(0, std::integral_constant<int, kBlock + H>());
        } else {
            for (int e = 0; e < p.count + H; ++e) tokens(e, std::integral_constant<int, 1>());
        }
    }
#pragma unroll
    for (int k = 0; k < W + 1; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) a.parts[((int64_t)run * (W + 1) + k) * a.D + d + i] = k < W ? dw[k < W ? k : 0][i] : db[i];
}

// Sums over the runs, [runs, W + 1, D] -> dweight [D, W] and dbias [D].  A workgroup takes 64 columns; its waves the runs in turn.
__global__ __launch_bounds__(kThreads) void k_conv_packed_sum(ConvArgs a, int W, float* dweight, float* dbias)
{
    __shared__ float part[kWaves][64];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int64_t n = (int64_t)(W + 1) * a.D, col = (int64_t)blockIdx.x * 64 + lane;
    float s[4] = {};
    if (col < n && a.ix.good()) {
        int r = wave;
        for (; r + 3 * kWaves < a.runs; r += 4 * kWaves) {
#pragma unroll
            for (int q = 0; q < 4; ++q) s[q] += a.parts[(r + q * kWaves) * n + col];
        }
        for (; r < a.runs; r += kWaves) s[0] += a.parts[r * n + col];
    }
    part[wave][lane] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (wave != 0 || col >= n) return;
    float sum = 0.f;
    for (int w = 0; w < kWaves; ++w) sum += part[w][lane];
    const int k = (int)(col / a.D), d = (int)(col % a.D);
    if (k < W) dweight[(int64_t)d * W + k] = sum;
    else if (dbias) dbias[d] = sum;
}

// The widest vector of channels, at most `most`, that D is whole numbers of (a lane's channels are all there or none is).
template <int MOST, typename F> void by_width(int64_t D, F&& f)
{
    if constexpr (MOST >= 8) {
        if (D % 8 == 0) return f(std::integral_constant<int, 8>());
    }
    if constexpr (MOST >= 4) {
        if (D % 4 == 0) return f(std::integral_constant<int, 4>());
    }
    if (D % 2 == 0) return f(std::integral_constant<int, 2>());
    return f(std::integral_constant<int, 1>());
}
template <typename F> void by_taps(int W, F&& f)
{
    if (W == 1) f(std::integral_constant<int, 1>());
    else if (W == 2) f(std::integral_constant<int, 2>());
    else if (W == 3) f(std::integral_constant<int, 3>());
    else f(std::integral_constant<int, 4>());
}

// Runs of pieces the backward pass is cut into: about 2048 waves fill the GPU, and more runs are more partial sums to add up.
int64_t runs_of(int64_t pieces, int64_t groups, int32_t* run)
{
    const int64_t want = (2048 + groups - 1) / groups;
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
        by_width<16 / (int)sizeof(T)>(D, [&](auto v) {
            constexpr int V = decltype(v)::value;
            a.groups = (int32_t)((D + 64 * V - 1) / (64 * V));
            const int64_t grid = (l.max_blocks + kWaves - 1) / kWaves * a.groups;
            fits = grid <= INT32_MAX;
            if (!fits) return;
            by_taps(W, [&](auto w) { k_conv_packed<T, V, decltype(w)::value><<<(unsigned)grid, kThreads, 0, stream>>>(a); });
        });
    });
    if (!fits) return fail(COREY_ESHAPE, "%s: T * D is too large", who);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? corey::hip_fail(e, "corey_conv_packed launch") : COREY_OK;
}

namespace {
// Channels of a lane in the backward pass: 8 bytes of 16-bit values, 16 of binary32 (its window of rows takes the registers).
template <typename F> void by_backward_width(corey_dtype dt, int64_t D, F&& f)
{
    by_type(dt, [&](auto t) { by_width<4>(D, [&](auto v) { f(t, v); }); });
}
int64_t backward_width(int64_t D) { return D % 4 == 0 ? 4 : D % 2 == 0 ? 2 : 1; }
}  // namespace

extern "C" size_t corey_conv_packed_bwd_workspace(const corey_pack* pack, int64_t D, int32_t W)
{
    Index ix;
    if (W < 1 || W > COREY_MAX_CONV || D < 1 || D > COREY_PACK_MAX_CHANNELS || index_of("corey_conv_packed_bwd_workspace", pack, &ix)) return 0;
    const Layout l = layout(pack->S, pack->T, pack->tile);
    const int64_t wide = 64 * backward_width(D);
    int32_t run;
    return (size_t)(runs_of(l.max_blocks, (D + wide - 1) / wide, &run) * (W + 1) * D) * 4;
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
    const int64_t wide = 64 * backward_width(D);
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
    a.groups = (int32_t)((D + wide - 1) / wide);
    a.runs = (int32_t)runs_of(l.max_blocks, a.groups, &a.run);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const unsigned grid = (unsigned)((a.runs + kWaves - 1) / kWaves * a.groups);
    by_backward_width(dt, D, [&](auto t, auto v) {
        by_taps(W, [&](auto w) {
            k_conv_packed_bwd<decltype(t), decltype(v)::value, decltype(w)::value><<<grid, kThreads, 0, stream>>>(a);
        });
    });
    k_conv_packed_sum<<<(unsigned)(((W + 1) * D + 63) / 64), kThreads, 0, stream>>>(a, W, dweight, dbias);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? corey::hip_fail(e, "corey_conv_packed_bwd launch") : COREY_OK;
}
