"""Packed batches as a program uses them: prompts, then tokens one by one; captured and replayed; on several streams; with memory that
is no index; far apart in memory.  And what the binding refuses."""
import numpy as np
import pytest
import torch

import packed_ref as ref
import paper_2604_10597_amd as corey
from packed_util import Batch, f64, rounded
from paper_2604_10597_amd import binding

pytestmark = pytest.mark.gpu

DEV = "cuda"


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def scan_kw(b):
    return dict(Dv=b.Dv, z=b.z, delta_bias=b.bias)


# ------------------------------------------------------------------------------------------- prompts and generation
def test_prompts_then_tokens_are_one_long_sequence():
    """Three prompts of one call, each continued token by token, the second by two continuations of the same state: convolution and scan
    equal those of the whole sequences."""
    D, N, W, more = 96, 16, 4, 5
    prompts = [20, 37, 1]
    follow = [0, 1, 1, 2]                                        # the prompt that each continuation comes from
    g = np.random.default_rng(11)
    w64 = (g.uniform(-1, 1, (D, W)) / 2).astype(np.float32).astype(np.float64)
    b64 = (g.uniform(-1, 1, D) / 2).astype(np.float32).astype(np.float64)
    w, bias = torch.from_numpy(w64.astype(np.float32)).to(DEV), torch.from_numpy(b64.astype(np.float32)).to(DEV)
    batch = Batch(prompts, D, N, "f32", seed=1)
    later = [Batch([1] * len(follow), D, N, "f32", seed=20 + k) for k in range(more)]
    for x in later:                                              # one layer: the same A, D and bias
        x.A, x.A64, x.Dv, x.Dv64, x.bias, x.bias64 = batch.A, batch.A64, batch.Dv, batch.Dv64, batch.bias, batch.bias64
    xs, xs64 = rounded(g.standard_normal((sum(prompts), D)), "f32")
    xl = [rounded(g.standard_normal((len(follow), D)), "f32") for _ in range(more)]

    conv_pool = torch.zeros((8, D, W - 1), device=DEV)
    pool = torch.full((8, D, N), 7.0, device=DEV)
    pack = corey.corey_pack_plan(ints(*prompts), sum(prompts), 16)
    none = ints(-1, -1, -1)
    u = corey.corey_conv_packed(xs.to(DEV), w, bias, pack, state=conv_pool, slots=none, slots_out=ints(5, 0, 3))
    y = corey.corey_scan_packed(u, batch.delta, batch.A, batch.B, batch.C, pack, state=pool, slots=none, slots_out=ints(5, 0, 3), **scan_kw(batch))
    read, write = ints(5, 0, 0, 3), ints(5, 1, 2, 3)             # the second prompt's state begins two sequences
    us, ys = [], []
    ones = corey.corey_pack_plan(ints(1, 1, 1, 1), 4, 16)
    for k in range(more):
        us.append(corey.corey_conv_packed(xl[k][0].to(DEV), w, bias, ones, state=conv_pool, slots=read, slots_out=write))
        ys.append(corey.corey_scan_packed_step(pool, read, us[k], later[k].delta, batch.A, later[k].B, later[k].C, slots_out=write, **scan_kw(later[k])))
        read = write
    assert torch.equal(pool[4], torch.full_like(pool[4], 7.0)) and torch.equal(pool[6:], torch.full_like(pool[6:], 7.0))

    starts = np.concatenate([[0], np.cumsum(prompts)])
    for s, p in enumerate(follow):
        rows = slice(starts[p], starts[p + 1])
        cat = lambda first, rest: np.concatenate([first[rows]] + [r[s:s + 1] for r in rest])
        x64 = cat(xs64, [v for _, v in xl])
        out, bound, _ = ref.conv(x64, w64, b64, np.zeros((D, W - 1)), "f32")
        got_u = cat(f64(u), [f64(v) for v in us])
        ref.check(got_u, out, bound, f"u of continuation {s}")
        r = ref.Scan(got_u, cat(batch.delta64, [v.delta64 for v in later]), batch.A64, cat(batch.B64, [v.B64 for v in later]),
                     cat(batch.C64, [v.C64 for v in later]), batch.Dv64, cat(batch.z64, [v.z64 for v in later]), batch.bias64, True,
                     np.zeros((D, N)), 16)
        ref.check(cat(f64(y), [f64(v) for v in ys]), *r.forward("f32"), f"y of continuation {s}")
        ref.check(f64(pool[write[s]]), *r.last(), f"state of continuation {s}")


@pytest.mark.parametrize("cut", [1, 15, 16, 17, 50])
def test_a_prompt_in_two_calls(cut):
    """A prompt cut anywhere and carried on by its slots gives what one call gives."""
    b = Batch([70], 80, 16, "bf16", seed=cut)
    whole, halves = torch.zeros((1, 80, 16), device=DEV), torch.zeros((1, 80, 16), device=DEV)
    pack = corey.corey_pack_plan(ints(70), 70, 32)
    y = corey.corey_scan_packed(b.u, b.delta, b.A, b.B, b.C, pack, state=whole, slots=ints(-1), slots_out=ints(0), **scan_kw(b))
    r = b.scan(0, None, True, 32)
    ref.check(f64(y), *r.forward("bf16"), "y of one call")
    out, slots = [], ints(-1)
    for f, e in ((0, cut), (cut, 70)):
        p = corey.corey_pack_plan(ints(e - f), e - f, 32)
        out.append(corey.corey_scan_packed(b.u[f:e], b.delta[f:e], b.A, b.B[f:e], b.C[f:e], p, Dv=b.Dv, z=b.z[f:e], delta_bias=b.bias,
                                           state=halves, slots=slots, slots_out=ints(0)))
        slots = ints(0)
    ref.check(f64(torch.cat(out)), *r.forward("bf16"), "y of two calls")
    for pool in (whole, halves):
        ref.check(f64(pool[0]), *r.last(), "state")


def test_one_state_begins_several_sequences():
    b = Batch([20, 20, 40, 3], 70, 16, "f32", seed=2)
    pool64 = np.random.default_rng(3).standard_normal((6, 70, 16)).astype(np.float32)
    pool = torch.from_numpy(pool64).to(DEV)
    pack = corey.corey_pack_plan(b.lens(), b.T, 16)
    y = corey.corey_scan_packed(b.u, b.delta, b.A, b.B, b.C, pack, state=pool, slots=ints(5, 5, 5, 5), slots_out=ints(0, 3, 1, -1), **scan_kw(b))
    for s, slot in enumerate((0, 3, 1, None)):
        f, e = b.spans[s]
        r = b.scan(s, pool64[5].astype(np.float64), True, 16)
        ref.check(f64(y[f:e]), *r.forward("f32"), f"y of {s}")
        if slot is not None:
            ref.check(f64(pool[slot]), *r.last(), f"state of {s}")
    for k in (2, 4, 5):
        assert np.array_equal(pool[k].cpu().numpy(), pool64[k])


def test_long_tiles():
    b = Batch([2100, 5, 2048], 33, 16, "f32", seed=9)
    pack = corey.corey_pack_plan(b.lens(), b.T, 2048)
    y = corey.corey_scan_packed(b.u, b.delta, b.A, b.B, b.C, pack, **scan_kw(b))
    for s, (f, e) in enumerate(b.spans):
        ref.check(f64(y[f:e]), *b.scan(s, None, True, 2048).forward("f32"), f"y of {s}")


# ------------------------------------------------------------------------------------------- training
def test_a_layer_trained_on_documents():
    """Convolution and scan forward, both backward, as a training step runs them: the gradients of x, the taps and the scan's inputs."""
    lengths, D, N, W = [50, 3, 0, 100], 72, 16, 4
    b = Batch(lengths, D, N, "f32", seed=6)
    g = np.random.default_rng(5)
    x, x64 = rounded(g.standard_normal((b.T, D)), "f32")
    w64 = (g.uniform(-1, 1, (D, W)) / 2).astype(np.float32).astype(np.float64)
    w, x = torch.from_numpy(w64.astype(np.float32)).to(DEV), x.to(DEV)
    pack = corey.corey_pack_plan(b.lens(), b.T, corey.corey_pack_tile(len(lengths), b.T, D, N, backward=True))
    u = corey.corey_conv_packed(x, w, None, pack)
    y = corey.corey_scan_packed(u, b.delta, b.A, b.B, b.C, pack, **scan_kw(b))
    grads = corey.corey_scan_packed_bwd(u, b.delta, b.A, b.B, b.C, pack, b.dy, **scan_kw(b))
    dx, dw, db = corey.corey_conv_packed_bwd(x, w, None, grads["du"], pack)
    u64, du64 = f64(u), f64(grads["du"])
    sums = [np.zeros((D, W)), np.zeros((D, W))]
    for s, (f, e) in enumerate(b.spans):
        if e == f:
            continue
        out, bound, _ = ref.conv(x64[f:e], w64, np.zeros(D), np.zeros((D, W - 1)), "f32")
        ref.check(u64[f:e], out, bound, "u")
        r = ref.Scan(u64[f:e], b.delta64[f:e], b.A64, b.B64[f:e], b.C64[f:e], b.Dv64, b.z64[f:e], b.bias64, True, np.zeros((D, N)), pack.tile)
        ref.check(f64(y[f:e]), *r.forward("f32"), "y")
        v, err = r.backward(b.dy64[f:e], 12, b.T // 16 + 4)["du"]
        ref.check(du64[f:e], v, ref.stored(v, err, "f32"), "du")
        (rx, bx), rw, _ = ref.conv_bwd(x64[f:e], w64, np.zeros(D), du64[f:e], "f32", more=b.T // 16 + 64)
        ref.check(f64(dx[f:e]), rx, bx, "dx")
        sums[0] += rw[0]
        sums[1] += rw[1]
    ref.check(f64(dw), sums[0], sums[1], "dweight")


def test_no_tokens_no_gradients():
    b = Batch([0, 0], 40, 16, "f32", T=6)
    pack = corey.corey_pack_plan(b.lens(), 6, 16)
    g = corey.corey_scan_packed_bwd(b.u, b.delta, b.A, b.B, b.C, pack, b.dy, **scan_kw(b))
    for k in ("dA", "dD", "ddelta_bias"):
        assert (g[k] == 0).all(), k
    _, dw, db = corey.corey_conv_packed_bwd(b.u, torch.ones(40, 4, device=DEV), None, b.dy, pack)
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_lies_behind_the_last_sequence_is_not_read(dtype):
    """NaN in the rows behind the last sequence, and infinities: every result is bit for bit what it is without them."""
    lengths, T, D, N = [17, 0, 40], 70, 72, 16
    n = sum(lengths)
    runs = []
    for filler in (0.0, float("nan"), float("inf")):
        b = Batch(lengths, D, N, dtype, T=T, seed=3)
        for t in (b.u, b.delta, b.B, b.C, b.z, b.dy):
            t[n:] = filler
        pack = corey.corey_pack_plan(b.lens(), T, 32)
        pool = torch.zeros((3, D, N), device=DEV)
        y = corey.corey_scan_packed(b.u, b.delta, b.A, b.B, b.C, pack, state=pool, slots=ints(-1, -1, -1), slots_out=ints(0, 1, 2), **scan_kw(b))
        w = torch.linspace(-1, 1, 4 * D, device=DEV).reshape(D, 4)
        conv_pool = torch.zeros((3, D, 3), device=DEV, dtype=b.u.dtype)
        u = corey.corey_conv_packed(b.u, w, None, pack, state=conv_pool, slots=ints(0, 1, 2))
        dx, dw, db = corey.corey_conv_packed_bwd(b.u, w, None, b.dy, pack)
        g = corey.corey_scan_packed_bwd(b.u, b.delta, b.A, b.B, b.C, pack, b.dy, **scan_kw(b))
        runs.append([y[:n], pool, u[:n], conv_pool, dx[:n], dw, db] + [g[k][:n] if k in ("du", "ddelta", "dz", "dB", "dC") else g[k] for k in sorted(g)])
    for other in runs[1:]:
        for a, c in zip(runs[0], other):
            assert torch.isfinite(a).all() and torch.equal(a, c)


def test_a_sequence_of_nan_keeps_it_to_itself():
    b = Batch([30, 20, 33], 72, 16, "f32", seed=8)
    pack = corey.corey_pack_plan(b.lens(), b.T, 16)
    names = ("du", "ddelta", "dz", "dB", "dC")

    def run():
        pool = torch.zeros((3, 72, 16), device=DEV)
        y = corey.corey_scan_packed(b.u, b.delta, b.A, b.B, b.C, pack, state=pool, slots=ints(0, 1, 2), **scan_kw(b))
        w = torch.linspace(-1, 1, 4 * 72, device=DEV).reshape(72, 4)
        g = corey.corey_scan_packed_bwd(b.u, b.delta, b.A, b.B, b.C, pack, b.dy, **scan_kw(b))
        return [y, corey.corey_conv_packed(b.u, w, None, pack), corey.corey_conv_packed_bwd(b.u, w, None, b.dy, pack)[0]] + [g[k] for k in names], pool
    clean, pool = run()
    for t in (b.u, b.dy):
        t[30:50] = float("nan")
    dirty, pool2 = run()
    for a, c in zip(clean, dirty):
        assert torch.equal(a[:30], c[:30]) and torch.equal(a[50:], c[50:]) and not torch.isfinite(c[30:50]).any(dim=1).all()
    assert torch.equal(pool[0], pool2[0]) and torch.equal(pool[2], pool2[2])


@pytest.mark.parametrize("N, tile", [(21, 16), (21, 64), (50, 48), (35, 32), (127, 32), (3, 64)])
def test_states_that_fill_no_wave(N, tile):
    """Forward and backward with numbers of states that leave a wave's last group of four, its last pair or a whole wave unfilled."""
    lengths = [40, 1, 0, 70, 16]
    b = Batch(lengths, 67, N, "f32", seed=N)
    pack = corey.corey_pack_plan(b.lens(), b.T, tile)
    y = corey.corey_scan_packed(b.u, b.delta, b.A, b.B, b.C, pack, **scan_kw(b))
    g = corey.corey_scan_packed_bwd(b.u, b.delta, b.A, b.B, b.C, pack, b.dy, **scan_kw(b))
    sums = {}
    for s, (f, e) in enumerate(b.spans):
        if e == f:
            continue
        r = b.scan(s, None, True, tile)
        ref.check(f64(y[f:e]), *r.forward("f32"), "y")
        for k, (v, err) in r.backward(b.dy64[f:e], 12, b.T // 16 + 5).items():
            if k in ("dA", "dD", "ddelta_bias"):
                old = sums.get(k, (0.0, 0.0))
                sums[k] = (old[0] + v, old[1] + err)
            else:
                ref.check(f64(g[k][f:e]), v, ref.stored(v, err, "f32"), k)
    for k, (v, err) in sums.items():
        ref.check(f64(g[k]), v, err + ref.TINY["f32"], k)


def test_growing_states_from_zero():
    """Step sizes below 0 (no softplus): over the first block the decays multiply to more than binary32 holds, but the state there is 0 (B is),
    so nothing of it may show."""
    D, N, n = 8, 4, 33
    b = Batch([n], D, N, "f32", seed=3, gated=False, skip=False, bias=False)
    b.A64 = -np.ones((D, N))
    delta = np.full((n, D), 0.1)
    delta[:16] = -89.2 / 16
    b.delta, b.delta64 = rounded(delta, "f32")
    bm = b.B64.copy()
    bm[:16] = 0.0
    b.B, b.B64 = rounded(bm, "f32")
    b.dy, b.dy64 = rounded(1e-6 * b.dy64, "f32")
    to = lambda t: t.to(DEV)
    pack = corey.corey_pack_plan(b.lens(), n, 48)
    g = corey.corey_scan_packed_bwd(b.u, to(b.delta), to(torch.from_numpy(b.A64.astype(np.float32))), to(b.B), b.C, pack, to(b.dy), delta_softplus=False)
    back = b.scan(0, None, False, 48).backward(b.dy64, 12, 4)
    for k in ("du", "ddelta", "dB", "dC"):
        ref.check(f64(g[k]), back[k][0], ref.stored(*back[k], "f32"), k)
    ref.check(f64(g["dA"]), back["dA"][0], back["dA"][1] + ref.TINY["f32"], "dA")
    pool = torch.zeros(1, D, N, device=DEV)                      # and over a tile, from a state of 0
    y = corey.corey_scan_packed(b.u, to(b.delta), to(torch.from_numpy(b.A64.astype(np.float32))), to(b.B), b.C,
                                corey.corey_pack_plan(b.lens(), n, 16), delta_softplus=False, state=pool, slots=ints(0))
    r = b.scan(0, None, False, 16)
    ref.check(f64(y), *r.forward("f32"), "y")
    ref.check(f64(pool[0]), *r.last(), "state")


# ------------------------------------------------------------------------------------------- graphs and streams
def test_two_graphs_replayed_in_turn():
    """Index, convolution, scan and gradients in one graph, generation in another that works on the same pools; replayed in turn with new
    lengths and inputs, eager work between; every replay is bit for bit what eager calls give."""
    D, N, W, S, T = 80, 16, 4, 5, 128
    g = torch.Generator(device=DEV).manual_seed(1)
    rnd = lambda *s: torch.randn(*s, device=DEV, generator=g)
    A, Dv, bias, w = -torch.exp(0.3 * rnd(D, N)), rnd(D), rnd(D) - 2, rnd(D, W)
    lens = torch.zeros(S, dtype=torch.int32, device=DEV)
    x, delta, z, dy, B, C = rnd(T, D), rnd(T, D), rnd(T, D), rnd(T, D), rnd(T, N), rnd(T, N)
    sx, sd, sz, sB, sC = rnd(S, D), rnd(S, D), rnd(S, D), rnd(S, N), rnd(S, N)
    slots = ints(0, 1, 2, 3, 4)
    one = torch.ones(S, dtype=torch.int32, device=DEV)
    tile = 32

    def prompts(pools):
        pack = corey.corey_pack_plan(lens, T, tile)
        u = corey.corey_conv_packed(x, w, None, pack, state=pools[0], slots=slots)
        y = corey.corey_scan_packed(u, delta, A, B, C, pack, Dv=Dv, z=z, delta_bias=bias, state=pools[1], slots=slots)
        grads = corey.corey_scan_packed_bwd(u, delta, A, B, C, pack, dy, Dv=Dv, z=z, delta_bias=bias)
        return [pack.starts, u, y, *corey.corey_conv_packed_bwd(x, w, None, grads["du"], pack), *(grads[k] for k in sorted(grads))]

    def tokens(pools):
        u = corey.corey_conv_packed(sx, w, None, corey.corey_pack_plan(one, S, 16), state=pools[0], slots=slots)
        return [corey.corey_scan_packed_step(pools[1], slots, u, sd, A, sB, sC, Dv=Dv, z=sz, delta_bias=bias)]

    make = lambda: [torch.zeros(6, D, W - 1, device=DEV), torch.zeros(6, D, N, device=DEV)]
    captured, eager = make(), make()
    lens.copy_(ints(20, 0, 1, 40, 33))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        prompts(make())
        tokens(make())
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for path in (prompts, tokens):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = path(captured)
        graphs.append((graph, out, path))
    for t in captured:
        t.zero_()
    at = lambda i, t: t[:sum(new)] if i == 0 and t.dim() == 2 and t.shape[0] == T else t      # (rows behind the last sequence: not written)
    for new in ([20, 0, 1, 40, 33], [1, 1, 1, 1, 1], [0, 0, 128, 0, 0], [64, 16, 17, 15, 9]):
        lens.copy_(ints(*new))
        for t in (x, delta, z, dy, B, C, sx, sd, sz, sB, sC):
            t.copy_(torch.randn(t.shape, device=DEV, generator=g))
        for i, (graph, out, path) in enumerate(graphs):
            graph.replay()
            torch.cuda.synchronize()
            for a, c in zip(out, path(eager)):
                assert torch.equal(at(i, a), at(i, c)), new
            for a, c in zip(captured, eager):
                assert torch.equal(a, c), (new, "pools")
            (x @ x.T).sum().item()


def test_streams():
    """On a stream that is not the default one, behind work of its own; and on two streams at once with one index between them."""
    batches = [Batch([300, 40, 5], 256, 16, "bf16", seed=s) for s in (1, 2)]
    pack = corey.corey_pack_plan(batches[0].lens(), 345, 48)
    run = lambda b: [corey.corey_scan_packed(b.u, b.delta, b.A, b.B, b.C, pack, **scan_kw(b)),
                     *corey.corey_scan_packed_bwd(b.u, b.delta, b.A, b.B, b.C, pack, b.dy, **scan_kw(b)).values()]
    want = [run(b) for b in batches]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in batches]
    got = []
    for b, st in zip(batches, streams):
        with torch.cuda.stream(st):
            late = torch.randn(1024, 1024, device=DEV)
            for _ in range(20):
                late = late @ late * 1e-2
            b.u.copy_(b.u + 0 * late[0, 0].nan_to_num(0, 0, 0).to(b.u.dtype))
            got.append(run(b))
    torch.cuda.synchronize()
    for a, c in zip(want, got):
        for p, q in zip(a, c):
            assert torch.equal(p, q)


@pytest.mark.parametrize("lengths, T, D, N, tile", [([40, 1, 0, 70, 16], 127, 67, 16, 16), ([17], 17, 300, 16, 64), ([64, 64], 128, 130, 40, 32), ([5, 5, 5], 16, 33, 128, 16), ([500], 503, 64, 7, 48)])
def test_a_workspace_of_the_callers(lengths, T, D, N, tile):
    """Workspaces, and the table, of exactly the sizes asked for, with whatever they hold: the same results, nothing written behind them."""
    b = Batch(lengths, D, N, "f32", T=T, seed=1)
    L, room = binding.lib(), 4096

    def memory(n):
        whole = torch.randint(0, 256, (n + room,), dtype=torch.uint8, device=DEV)
        return whole, whole[n:].clone()
    guards = []

    def exactly(n):
        whole, behind = memory(n)
        guards.append((whole[n:], behind))
        return whole[:n]
    table = exactly(L.corey_pack_bytes(len(lengths), T, tile)).view(torch.int32)
    pack, other = corey.corey_pack_plan(b.lens(), T, tile, table=table), corey.corey_pack_plan(b.lens(), T, tile)
    n = sum(lengths)
    for x, y in zip((pack.starts, pack.seq, pack.tiles, pack.blocks), (other.starts, other.seq, other.tiles, other.blocks)):
        assert torch.equal(x, y)
    y = corey.corey_scan_packed(b.u, b.delta, b.A, b.B, b.C, pack, workspace=exactly(L.corey_scan_packed_workspace(pack, D, N)), **scan_kw(b))
    assert torch.equal(y[:n], corey.corey_scan_packed(b.u, b.delta, b.A, b.B, b.C, other, **scan_kw(b))[:n])
    g = corey.corey_scan_packed_bwd(b.u, b.delta, b.A, b.B, b.C, pack, b.dy, workspace=exactly(L.corey_scan_packed_bwd_workspace(pack, D, N)), **scan_kw(b))
    for k, v in corey.corey_scan_packed_bwd(b.u, b.delta, b.A, b.B, b.C, other, b.dy, **scan_kw(b)).items():
        assert torch.equal(g[k][:n], v[:n]) if k in ("du", "ddelta", "dz", "dB", "dC") else torch.equal(g[k], v), k
    w = torch.linspace(-1, 1, 4 * D, device=DEV).reshape(D, 4)
    mine = corey.corey_conv_packed_bwd(b.u, w, None, b.dy, pack, workspace=exactly(L.corey_conv_packed_bwd_workspace(pack, D, 4)))
    dx, dw, db = corey.corey_conv_packed_bwd(b.u, w, None, b.dy, other)
    assert torch.equal(mine[0][:n], dx[:n]) and torch.equal(mine[1], dw) and torch.equal(mine[2], db)
    for now, before in guards:
        assert torch.equal(now, before)


# ------------------------------------------------------------------------------------------- memory that is no index
@pytest.mark.parametrize("kind", ["zeros", "noise", "other sizes", "other tile"])
def test_memory_that_is_no_index_is_not_followed(kind):
    b = Batch([20, 30, 14], 64, 16, "f32", seed=1)
    pack = corey.corey_pack_plan(b.lens(), 64, 32)
    if kind == "zeros":
        pack.table.zero_()
    elif kind == "noise":
        pack.table.random_(-2**31, 2**31 - 1)
    else:                                                        # another index was built in the same memory
        corey.corey_pack_plan(b.lens() if kind == "other tile" else ints(9, 9), 64 if kind == "other tile" else 20, 64 if kind == "other tile" else 32, table=pack.table)
    nine = lambda *s: torch.full(s, 9.0, device=DEV)
    y, u, pool = nine(64, 64), nine(64, 64), nine(3, 64, 16)
    corey.corey_scan_packed(b.u, b.delta, b.A, b.B, b.C, pack, state=pool, slots=ints(0, 1, 2), y=y, **scan_kw(b))
    conv_pool, w = nine(3, 64, 3), nine(64, 4)
    corey.corey_conv_packed(b.u, w, None, pack, state=conv_pool, slots=ints(0, 1, 2), u=u)
    out = dict(du=nine(64, 64), ddelta=nine(64, 64), dz=nine(64, 64), dB=nine(64, 16), dC=nine(64, 16), dA=nine(64, 16), dD=nine(64), ddelta_bias=nine(64))
    corey.corey_scan_packed_bwd(b.u, b.delta, b.A, b.B, b.C, pack, b.dy, out=out, **scan_kw(b))
    dx, dw, db, ws = nine(64, 64), nine(64, 4), nine(64), nine(1 << 16)
    rc = binding.lib().corey_conv_packed_bwd(b.u.data_ptr(), 64, w.data_ptr(), None, b.dy.data_ptr(), 64, pack, dx.data_ptr(), 64, dw.data_ptr(),
                                             db.data_ptr(), binding.COREY_F32, 64, 4, ws.data_ptr(), ws.nbytes, torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    for t in (y, u, pool, conv_pool, dx, dw, db, *out.values()):
        assert (t == 9.0).all()


# ------------------------------------------------------------------------------------------- far apart in memory
def test_a_pool_beyond_32_bits():
    """Slots whose states lie more than 2^31 values and 2^33 bytes into the pool."""
    D, N = 2048, 16
    n = (2**31 // (D * N)) + 40
    pool = torch.empty((n, D, N), device=DEV)
    conv_pool = torch.empty((2**31 // (D * 3) + 40, D, 3), device=DEV, dtype=torch.bfloat16)
    b = Batch([1, 1], D, N, "bf16", seed=4)
    last, conv_last = n - 1, conv_pool.shape[0] - 1
    g = np.random.default_rng(7)
    first = g.standard_normal((2, D, N)).astype(np.float32)
    pool[last], pool[3] = torch.from_numpy(first[0]).to(DEV), torch.from_numpy(first[1]).to(DEV)
    y = corey.corey_scan_packed_step(pool, ints(last, 3), b.u, b.delta, b.A, b.B, b.C, slots_out=ints(last - 1, 3), **scan_kw(b))
    pack = corey.corey_pack_plan(b.lens(), 2, 16)
    y2 = corey.corey_scan_packed(b.u, b.delta, b.A, b.B, b.C, pack, state=pool, slots=ints(last, 3), slots_out=ints(last - 2, -1), **scan_kw(b))
    for s, slot in ((0, last - 1), (1, 3)):
        r = b.scan(s, first[s].astype(np.float64), True, 16)
        ref.check(f64(y[s:s + 1]), *r.forward("bf16"), "y")
        ref.check(f64(pool[slot]), *r.last(), "state")
        if s == 0:
            ref.check(f64(y2[:1]), *r.forward("bf16"), "y")
            ref.check(f64(pool[last - 2]), *r.last(), "state")
    old, old64 = rounded(g.standard_normal((D, 3)), "bf16")
    conv_pool[conv_last] = old.to(DEV)
    w64 = (g.uniform(-1, 1, (D, 4)) / 2).astype(np.float32).astype(np.float64)
    u = corey.corey_conv_packed(b.u, torch.from_numpy(w64.astype(np.float32)).to(DEV), None, pack, state=conv_pool, slots=ints(conv_last, -1),
                                slots_out=ints(conv_last - 1, -1))
    out, bound, new = ref.conv(b.u64[:1], w64, np.zeros(D), old64, "bf16")
    ref.check(f64(u[:1]), out, bound, "u")
    assert np.array_equal(f64(conv_pool[conv_last - 1]), new)


def test_rows_beyond_32_bits():
    """A batch of more than 2^31 values; its last sequence is compared."""
    D, N, W = 8192, 16, 4
    tail = 21
    T = 2**31 // D + 60 + tail
    g = torch.Generator(device=DEV).manual_seed(2)
    rnd = lambda *s: torch.randn(*s, device=DEV, generator=g, dtype=torch.bfloat16)
    b = Batch([tail], D, N, "bf16", seed=5)
    rows = {}
    for k, wide in (("u", D), ("delta", D), ("dy", D), ("B", N), ("C", N)):
        rows[k] = rnd(T, wide)
        rows[k][T - tail:] = getattr(b, k)
    w64 = np.random.default_rng(1).uniform(-1, 1, (D, W)).astype(np.float32).astype(np.float64)
    w = torch.from_numpy(w64.astype(np.float32)).to(DEV)
    pack = corey.corey_pack_plan(ints(T - tail - 7, 7, tail), T, 64)
    y = corey.corey_scan_packed(rows["u"], rows["delta"], b.A, rows["B"], rows["C"], pack, delta_bias=b.bias)
    part = slice(0, 256)                                         # channels compared
    f = lambda a: a[:, part]
    r = ref.Scan(f(b.u64), f(b.delta64), b.A64[part], b.B64, b.C64, np.zeros(256), None, b.bias64[part], True, np.zeros((256, N)), 64)
    ref.check(f64(y[T - tail:, part]), *r.forward("bf16"), "y")
    del y
    grads = corey.corey_scan_packed_bwd(rows["u"], rows["delta"], b.A, rows["B"], rows["C"], pack, rows["dy"], delta_bias=b.bias)
    back = r.backward(f(b.dy64), 200, 1)
    for k in ("du", "ddelta"):
        ref.check(f64(grads[k][T - tail:, part]), back[k][0], ref.stored(*back[k], "bf16"), k)
    assert all(torch.isfinite(grads[k]).all() for k in ("dA", "dB", "dC", "ddelta_bias"))
    del grads
    u = corey.corey_conv_packed(rows["u"], w, None, pack)
    out, bound, _ = ref.conv(f(b.u64), w64[part], np.zeros(256), np.zeros((256, W - 1)), "bf16")
    ref.check(f64(u[T - tail:, part]), out, bound, "u")
    del u
    dx, _, _ = corey.corey_conv_packed_bwd(rows["u"], w, None, rows["dy"], pack)
    (rx, bx), _, _ = ref.conv_bwd(f(b.u64), w64[part], np.zeros(256), f(b.dy64), "bf16")
    ref.check(f64(dx[T - tail:, part]), rx, bx, "dx")


def test_rows_very_far_apart():
    """Rows 2^25 - 1 values apart, the most there is: 15 of them from the first are nearly 2^31 bytes away."""
    stride, D, N = 2**25 - 1, 70, 16
    b = Batch([18, 2], D, N, "f32", seed=6)
    mem = torch.empty(20 * stride + 4 * D, device=DEV)
    spread = lambda t, at: mem.as_strided(t.shape, (stride, 1), at).copy_(t)
    u, z = spread(b.u, 0), spread(b.z, D)
    y = mem.as_strided(b.u.shape, (stride, 1), 2 * D)
    pack = corey.corey_pack_plan(b.lens(), 20, 16)
    corey.corey_scan_packed(u, b.delta, b.A, b.B, b.C, pack, Dv=b.Dv, z=z, delta_bias=b.bias, y=y)
    for s, (f, e) in enumerate(b.spans):
        ref.check(f64(y[f:e]), *b.scan(s, None, True, 16).forward("f32"), "y")


# ------------------------------------------------------------------------------------------- refusals of the binding
def test_refusals():
    b = Batch([20, 12], 64, 16, "f32")
    pack = corey.corey_pack_plan(b.lens(), 32, 32)
    w, pool, conv_pool = torch.ones(64, 4, device=DEV), torch.zeros(2, 64, 16, device=DEV), torch.zeros(2, 64, 3, device=DEV)
    slots = ints(0, 1)
    scan = lambda **kw: corey.corey_scan_packed(**{**dict(u=b.u, delta=b.delta, A=b.A, Bm=b.B, Cm=b.C, pack=pack), **kw})
    conv = lambda **kw: corey.corey_conv_packed(**{**dict(x=b.u, weight=w, bias=None, pack=pack), **kw})
    bwd = lambda **kw: corey.corey_scan_packed_bwd(**{**dict(u=b.u, delta=b.delta, A=b.A, Bm=b.B, Cm=b.C, pack=pack, dy=b.dy), **kw})
    step = lambda **kw: corey.corey_scan_packed_step(**{**dict(state=pool, slots=slots, x=b.u[:2], delta=b.delta[:2], A=b.A, Bt=b.B[:2], Ct=b.C[:2]), **kw})
    cbwd = lambda **kw: corey.corey_conv_packed_bwd(**{**dict(x=b.u, weight=w, bias=None, du=b.dy, pack=pack), **kw})
    for call in (scan, conv, bwd, step, cbwd):
        call()
    half, wide = b.u.bfloat16(), torch.zeros(32, 128, device=DEV)
    stale = corey.corey_pack_plan(b.lens(), 32, 32)
    stale.table = stale.table.clone()
    bad = (TypeError, ValueError, AttributeError, binding.CoreyError)
    for call, kw in [
            (scan, dict(u=b.u.cpu())), (scan, dict(delta=half)), (scan, dict(u=b.u[:31])), (scan, dict(u=wide[:, ::2])), (scan, dict(u=b.u[:1].expand(32, 64))),
            (scan, dict(u=b.u.double())), (scan, dict(u=b.u.T)), (scan, dict(u=b.u[None])), (scan, dict(A=b.A.bfloat16())), (scan, dict(A=b.A[:63])), (scan, dict(A=b.A.T)),
            (scan, dict(Bm=b.B[:, :8])), (scan, dict(Cm=b.C.cpu())), (scan, dict(z=b.u[:, :32])), (scan, dict(Dv=torch.ones(63, device=DEV))),
            (scan, dict(delta_bias=torch.ones(64))), (scan, dict(pack=None)), (scan, dict(pack=stale)), (scan, dict(pack=corey.Pack())), (scan, dict(slots=slots)),
            (scan, dict(state=pool, slots=slots.long())), (scan, dict(state=pool, slots=ints(1))), (scan, dict(state=pool[:, :32], slots=slots)),
            (scan, dict(state=pool.half(), slots=slots)), (scan, dict(y=b.u)), (scan, dict(y=half)), (scan, dict(y=b.u[:5])), (scan, dict(workspace=ints(1))),
            (scan, dict(u=None)),
            (conv, dict(x=b.u.cpu())), (conv, dict(weight=torch.ones(64, 5, device=DEV))), (conv, dict(weight=w.half())), (conv, dict(weight=w[:32])),
            (conv, dict(bias=torch.ones(1, device=DEV))), (conv, dict(u=b.u)), (conv, dict(state=pool, slots=slots)), (conv, dict(state=conv_pool.half(), slots=slots)),
            (conv, dict(slots_out=slots)), (conv, dict(pack=stale)), (conv, dict(x=b.u.long())),
            (cbwd, dict(du=half)), (cbwd, dict(du=b.dy[:3])), (cbwd, dict(workspace=ints(1))), (cbwd, dict(weight=w.cpu())), (cbwd, dict(pack=stale)),
            (step, dict(state=None)), (step, dict(slots=None)), (step, dict(slots=ints(0, 1, 2))), (step, dict(state=pool[:, :, :8])), (step, dict(x=half[:2])),
            (step, dict(slots_out=slots.cpu())), (step, dict(y=b.u)), (step, dict(delta=b.delta)),
            (bwd, dict(dy=half)), (bwd, dict(dy=None)), (bwd, dict(out=dict(du=half))), (bwd, dict(out=dict(dA=half))), (bwd, dict(out=[])), (bwd, dict(out=dict(du=b.u))),
            (bwd, dict(workspace=ints(1))), (bwd, dict(pack=corey.corey_pack_plan(b.lens(), 32, 128))),
            (corey.corey_pack_plan, dict(lengths=b.lens().long(), T=32, tile=16)), (corey.corey_pack_plan, dict(lengths=b.lens().cpu(), T=32, tile=16)),
            (corey.corey_pack_plan, dict(lengths=b.lens(), T=32, tile=17)), (corey.corey_pack_plan, dict(lengths=b.lens(), T=0, tile=16)),
            (corey.corey_pack_plan, dict(lengths=b.lens(), T=32.0, tile=16)), (corey.corey_pack_plan, dict(lengths=b.lens(), T=32, tile=16, table=ints(1, 2, 3))),
            (corey.corey_pack_plan, dict(lengths=b.lens()[:0], T=32, tile=16))]:
        with pytest.raises(bad):
            call(**kw)
    torch.cuda.synchronize()
    for call in (scan, conv, bwd, step, cbwd):                   # and nothing was left behind
        call()
