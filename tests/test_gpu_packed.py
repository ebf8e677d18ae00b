"""Operators on packed batches on the GPU, against their 64-bit reference (packed_ref.py, which derives the bounds)."""
import numpy as np
import pytest
import torch

import packed_ref as ref
import paper_2604_10597_amd as corey
from packed_util import Batch, f64, rounded, rows

pytestmark = pytest.mark.gpu

RAGGED = [5, 0, 1, 40, 16, 17, 0, 129, 3, 2]


# ------------------------------------------------------------------------------------------- the index
@pytest.mark.parametrize("lengths, T, tile", [
    ([1], 1, 16), ([0], 3, 16), ([0, 0, 0], 1, 32), (RAGGED, 213, 16), (RAGGED, 230, 64), ([64] * 7, 448, 64),
    ([-5, 3, -1, 20], 23, 16),                       # lengths below 0 count as 0
    ([10, 20, 30, 5], 37, 16),                       # cut off inside the third sequence
    ([2**31 - 1, 2**31 - 1, 4], 50, 16),             # sums beyond 32 bits are cut off, too
    ([100, 1, 47, 48, 49], 245, 48), ([1] * 4096, 4096, 16), ([1] * 4097, 4097, 16), ([3, 0, 33] * 3000, 12 * 9000, 32), ([0] * 5000 + [2048], 2050, 2048),
])
def test_plan(lengths, T, tile):
    p = corey.corey_pack_plan(torch.tensor(lengths, dtype=torch.int32, device="cuda"), T, tile)
    for got, want, what in zip((p.starts, p.seq, p.tiles, p.blocks), ref.plan(lengths, T, tile), ("starts", "seq", "tiles", "blocks")):
        assert np.array_equal(got.cpu().numpy(), want), what
    head = p.table[:16].cpu().numpy()
    starts, _, tiles, blocks = ref.plan(lengths, T, tile)
    assert list(head[1:8]) == [len(lengths), T, tile, starts[-1], (tiles[:, 0] >= 0).sum(), (blocks[:, 0] >= 0).sum(), (np.diff(starts) > tile).sum()]


def test_plan_random():
    g = np.random.default_rng(3)
    for _ in range(12):
        S, tile = int(g.integers(1, 9000)), 16 * int(g.integers(1, 129))
        lengths = (g.integers(0, 60, S) * (g.random(S) < 0.8)).astype(np.int32)
        T = max(1, int(lengths.sum() * g.choice([0.5, 1.0, 1.1])))
        p = corey.corey_pack_plan(torch.from_numpy(lengths).cuda(), T, tile)
        for got, want in zip((p.starts, p.seq, p.tiles, p.blocks), ref.plan(lengths, T, tile)):
            assert np.array_equal(got.cpu().numpy(), want)


# ------------------------------------------------------------------------------------------- the convolution
def conv_inputs(D, W, n, dtype, lay, seed):
    g = np.random.default_rng(seed)
    x, x64 = rows(g.standard_normal((n, D)), dtype, lay)
    du, du64 = rows(g.standard_normal((n, D)), dtype, lay)
    w = (g.uniform(-1, 1, (D, W)) / W ** 0.5).astype(np.float32)
    b = (g.uniform(-1, 1, D) / W ** 0.5).astype(np.float32)
    return x, x64, du, du64, torch.from_numpy(w).cuda(), w.astype(np.float64), torch.from_numpy(b).cuda(), b.astype(np.float64)


@pytest.mark.parametrize("dtype, D, W, lay", [
    ("bf16", 512, 4, "plain"), ("bf16", 1000, 4, "wide"), ("f16", 130, 3, "odd"), ("f32", 67, 4, "odd"), ("f32", 256, 2, "wide"),
    ("bf16", 1, 4, "plain"), ("f16", 24, 1, "plain"), ("bf16", 513, 2, "plain")])
@pytest.mark.parametrize("in_place", [True, False])
def test_conv(dtype, D, W, lay, in_place):
    lengths, T = RAGGED, sum(RAGGED) + 7
    S = len(lengths)
    x, x64, _, _, w, w64, b, b64 = conv_inputs(D, W, T, dtype, lay, D + W)
    pool, pool64 = rounded(np.random.default_rng(1).standard_normal((2 * S * D, max(1, W - 1))), dtype)
    pool = pool.reshape(2 * S, D, -1)[:, :, :W - 1].contiguous().cuda()
    pool64 = pool64.reshape(2 * S, D, -1)[:, :, :W - 1].copy()
    order = np.random.default_rng(2).permutation(2 * S)
    read = order[:S].copy()
    read[4], read[7] = -1, 2 * S                                 # no state: from zero
    write = read if in_place else order[S:].copy()
    if not in_place:
        write[3] = -1                                            # the state is not kept
    ints = lambda v: torch.tensor(v.astype(np.int32)).cuda()
    u = torch.full((T, D), 9.0, dtype=x.dtype, device="cuda")
    pack = corey.corey_pack_plan(torch.tensor(lengths, dtype=torch.int32, device="cuda"), T, 32)
    corey.corey_conv_packed(x, w, b, pack, state=pool, slots=ints(read), slots_out=None if in_place else ints(write), u=u)
    expect = pool64.copy()
    for s, (f, e) in enumerate(ref.spans(lengths, T)):
        have = 0 <= read[s] < 2 * S
        st = pool64[read[s]] if have else np.zeros((D, W - 1))
        out, bound, new = ref.conv(x64[f:e], w64, b64, st, dtype)
        ref.check(f64(u[f:e]), out, bound, f"u of sequence {s}")
        if 0 <= write[s] < 2 * S and e > f:
            expect[write[s]] = new
    assert np.array_equal(f64(pool), expect), "states"           # inputs, moved: exact
    assert (u[sum(lengths):] == 9.0).all(), "rows behind the last sequence"


def test_conv_without_slots_and_bias():
    x, x64, _, _, w, w64, _, _ = conv_inputs(96, 4, 50, "f32", "plain", 5)
    pack = corey.corey_pack_plan(torch.tensor([20, 30], dtype=torch.int32, device="cuda"), 50, 16)
    u = corey.corey_conv_packed(x, w, None, pack)
    for f, e in ((0, 20), (20, 50)):
        out, bound, _ = ref.conv(x64[f:e], w64, np.zeros(96), np.zeros((96, 3)), "f32")
        ref.check(f64(u[f:e]), out, bound, "u")


@pytest.mark.parametrize("dtype, D, W, lay, lengths", [
    ("f32", 96, 4, "plain", RAGGED), ("bf16", 516, 4, "wide", RAGGED), ("f16", 130, 3, "odd", RAGGED), ("f32", 67, 2, "odd", RAGGED),
    ("bf16", 256, 1, "plain", RAGGED), ("f32", 300, 4, "plain", [1, 1, 2, 3, 0, 1]), ("f32", 8, 4, "plain", [1]), ("f32", 260, 4, "plain", [3000, 1, 700])])
def test_conv_gradients(dtype, D, W, lay, lengths):
    T = sum(lengths) + 3
    x, x64, du, du64, w, w64, b, b64 = conv_inputs(D, W, T, dtype, lay, 7 * D + W)
    pack = corey.corey_pack_plan(torch.tensor(lengths, dtype=torch.int32, device="cuda"), T, 64)
    dx, dw, db = corey.corey_conv_packed_bwd(x, w, b, du, pack)
    again = corey.corey_conv_packed_bwd(x, w, b, du, pack)
    n = sum(lengths)
    assert torch.equal(dx[:n], again[0][:n]) and torch.equal(dw, again[1]) and torch.equal(db, again[2]), "the order of the sums is fixed"
    sums = [np.zeros((D, W)), np.zeros((D, W)), np.zeros(D), np.zeros(D)]
    for f, e in ref.spans(lengths, T):
        if e == f:
            continue
        (rx, bx), rw, rb = ref.conv_bwd(x64[f:e], w64, b64, du64[f:e], dtype, more=sum(lengths) // 16 + 64)
        ref.check(f64(dx[f:e]), rx, bx, "dx")
        for i, v in enumerate((*rw, *rb)):
            sums[i] += v
    ref.check(f64(dw), sums[0], sums[1], "dweight")
    ref.check(f64(db), sums[2], sums[3], "dbias")


# ------------------------------------------------------------------------------------------- the scan
def run_scan(b, tile, softplus=True, in_place=True, seed=0):
    g = np.random.default_rng(seed)
    S = len(b.lengths)
    pool64 = g.standard_normal((2 * S, b.D, b.N)).astype(np.float32).astype(np.float64)
    pool = torch.from_numpy(pool64.astype(np.float32)).cuda()
    order = g.permutation(2 * S)
    read = order[:S].copy()
    if S > 2:
        read[2] = -1
    write = read if in_place else order[S:].copy()
    if not in_place and S > 3:
        write[3] = 2 * S + 7
    ints = lambda v: torch.tensor(v.astype(np.int32)).cuda()
    y = torch.full((b.T, b.D), 9.0, dtype=b.u.dtype, device="cuda")
    pack = corey.corey_pack_plan(b.lens(), b.T, tile)
    corey.corey_scan_packed(b.u, b.delta, b.A, b.B, b.C, pack, Dv=b.Dv, z=b.z, delta_bias=b.bias, delta_softplus=softplus, state=pool,
                            slots=ints(read), slots_out=None if in_place else ints(write), y=y)
    end = 0
    for s, (f, e) in enumerate(b.spans):
        end = e
        have = 0 <= read[s] < 2 * S
        keep = 0 <= write[s] < 2 * S
        if e == f:
            if keep:
                assert np.array_equal(f64(pool[write[s]]), pool64[write[s]]), "a sequence without tokens moved a state"
            continue
        r = b.scan(s, pool64[read[s]] if have else None, softplus, tile)
        ref.check(f64(y[f:e]), *r.forward(b.dtype), f"y of sequence {s}")
        if keep:
            ref.check(f64(pool[write[s]]), *r.last(), f"state of sequence {s}")
    touched = {int(w) for s, w in enumerate(write) if 0 <= w < 2 * S and b.spans[s][1] > b.spans[s][0]}
    for k in range(2 * S):
        if k not in touched:
            assert np.array_equal(f64(pool[k]), pool64[k]), f"slot {k} was not to be written"
    assert (y[end:] == 9.0).all(), "rows behind the last sequence"


@pytest.mark.parametrize("dtype, D, N, lay, tile", [
    ("f32", 128, 16, "plain", 16), ("f32", 130, 16, "wide", 32), ("f32", 67, 16, "odd", 64), ("bf16", 256, 16, "wide", 16),
    ("bf16", 129, 16, "odd", 128), ("f32", 64, 16, "plain", 48), ("f16", 192, 16, "odd", 16), ("f16", 1, 16, "plain", 16), ("f32", 2, 1, "plain", 16),
    ("f32", 70, 5, "odd", 16), ("bf16", 64, 8, "plain", 32), ("f32", 66, 24, "plain", 16), ("f16", 40, 64, "wide", 32),
    ("f32", 33, 100, "odd", 16), ("bf16", 64, 128, "plain", 64), ("f32", 96, 48, "plain", 256)])
@pytest.mark.parametrize("in_place", [True, False])
def test_scan(dtype, D, N, lay, tile, in_place):
    run_scan(Batch(RAGGED, D, N, dtype, T=sum(RAGGED) + 5, seed=D + N, lay=lay), tile, in_place=in_place)


@pytest.mark.parametrize("gated, skip, bias, softplus", [(False, True, True, True), (True, False, False, True), (False, False, False, False), (True, True, True, False)])
@pytest.mark.parametrize("N", [16, 20])
def test_scan_options(gated, skip, bias, softplus, N):
    b = Batch(RAGGED, 72, N, "f32", seed=4, gated=gated, skip=skip, bias=bias)
    if not softplus:                                             # step sizes are used as they are
        b.delta64 = np.abs(b.delta64) * 0.1
        b.delta, b.delta64 = rows(b.delta64, "f32", "plain")
        if bias:
            b.bias64 = np.abs(b.bias64) * 0.01
            b.bias64 = b.bias64.astype(np.float32).astype(np.float64)
            b.bias = torch.from_numpy(b.bias64.astype(np.float32)).cuda()
    run_scan(b, 32, softplus)


@pytest.mark.parametrize("lengths, T", [([1], 1), ([7], 7), ([8], 9), ([9], 9), ([15, 16, 17], 48), ([1] * 70, 70), ([0, 0], 4), ([300], 300), ([50, 60], 80)])
def test_scan_lengths(lengths, T):
    run_scan(Batch(lengths, 64, 16, "f32", T=T, seed=sum(lengths)), 16)


@pytest.mark.parametrize("N, dtype, lay", [(16, "bf16", "wide"), (16, "f32", "plain"), (5, "f16", "odd"), (64, "f32", "odd"), (256, "bf16", "plain"), (1, "f32", "plain")])
@pytest.mark.parametrize("S, D", [(1, 1), (9, 130), (33, 67)])
def test_step(N, dtype, lay, S, D):
    b = Batch([1] * S, D, N, dtype, seed=S + N, lay=lay)
    g = np.random.default_rng(1)
    pool64 = g.standard_normal((2 * S + 1, D, N)).astype(np.float32).astype(np.float64)
    for in_place in (True, False):
        pool = torch.from_numpy(pool64.astype(np.float32)).cuda()
        order = g.permutation(2 * S)
        read, write = order[:S].copy(), order[S:].copy()
        if S > 1:
            read[1] = -1
        if in_place:
            write = read
        ints = lambda v: torch.tensor(v.astype(np.int32)).cuda()
        y = corey.corey_scan_packed_step(pool, ints(read), b.u, b.delta, b.A, b.B, b.C, Dv=b.Dv, z=b.z, delta_bias=b.bias,
                                         slots_out=None if in_place else ints(write))
        expect = [None] * (2 * S + 1)
        for s in range(S):
            r = b.scan(s, pool64[read[s]] if read[s] >= 0 else None, True, 1)
            ref.check(f64(y[s:s + 1]), *r.forward(dtype), f"y of {s}")
            if write[s] >= 0:
                expect[write[s]] = r.last()
        for k, want in enumerate(expect):
            if want is None:
                assert np.array_equal(f64(pool[k]), pool64[k])
            else:
                ref.check(f64(pool[k]), *want, f"slot {k}")


# ------------------------------------------------------------------------------------------- the scan's gradients
def run_scan_bwd(b, tile, softplus=True):
    pack = corey.corey_pack_plan(b.lens(), b.T, tile)
    call = lambda: corey.corey_scan_packed_bwd(b.u, b.delta, b.A, b.B, b.C, pack, b.dy, Dv=b.Dv, z=b.z, delta_bias=b.bias, delta_softplus=softplus)
    g, again = call(), call()
    end = max(e for _, e in b.spans)
    for k in g:
        same = torch.equal(g[k][:end], again[k][:end]) if k in ("du", "ddelta", "dz", "dB", "dC") else torch.equal(g[k], again[k])
        assert same, f"{k}: the order of the sums is fixed"
    assert set(g) == {"du", "ddelta", "dA", "dB", "dC"} | ({"dz"} if b.z is not None else set()) | ({"dD"} if b.Dv is not None else set()) | (
        {"ddelta_bias"} if b.bias is not None else set())
    sums = {}
    for s, (f, e) in enumerate(b.spans):
        if e == f:
            continue
        r = b.scan(s, None, softplus, tile).backward(b.dy64[f:e], channel_adds=10 + b.D // 64, tile_adds=b.T // 16 + len(b.spans))
        for k, (v, err) in r.items():
            if k in ("dA", "dD", "ddelta_bias"):
                old = sums.get(k, (0.0, 0.0))
                sums[k] = (old[0] + v, old[1] + err)
            else:
                ref.check(f64(g[k][f:e]), v, ref.stored(v, err, b.dtype), f"{k} of sequence {s}")
    for k, (v, err) in sums.items():
        if k in g:
            ref.check(f64(g[k]), v, err + ref.TINY["f32"], k)


@pytest.mark.parametrize("dtype, D, N, lay, tile", [
    ("f32", 64, 16, "plain", 64), ("f32", 300, 16, "wide", 64), ("f32", 67, 16, "odd", 32), ("bf16", 256, 16, "wide", 64), ("f16", 129, 16, "odd", 16), ("f32", 64, 16, "plain", 48),
    ("f32", 1, 1, "plain", 16), ("f32", 70, 5, "odd", 64), ("f32", 66, 24, "plain", 64), ("bf16", 40, 64, "wide", 64), ("f32", 65, 40, "plain", 16),
    ("f32", 33, 100, "odd", 32), ("f16", 64, 128, "plain", 16)])
def test_scan_gradients(dtype, D, N, lay, tile):
    run_scan_bwd(Batch(RAGGED, D, N, dtype, T=sum(RAGGED) + 5, seed=D + N, lay=lay), tile)


@pytest.mark.parametrize("gated, skip, bias, softplus", [(False, True, True, True), (True, False, False, True), (False, False, False, False)])
@pytest.mark.parametrize("N", [16, 20])
def test_scan_gradients_options(gated, skip, bias, softplus, N):
    b = Batch(RAGGED, 72, N, "f32", seed=4, gated=gated, skip=skip, bias=bias)
    if not softplus:
        b.delta, b.delta64 = rows(np.abs(b.delta64) * 0.1, "f32", "plain")
    run_scan_bwd(b, 32, softplus)


@pytest.mark.parametrize("lengths, T", [([1], 1), ([7], 7), ([16], 17), ([17], 17), ([63, 64, 65], 192), ([1] * 70, 70), ([0, 3], 4), ([300], 300), ([50, 60], 80)])
def test_scan_gradients_lengths(lengths, T):
    run_scan_bwd(Batch(lengths, 64, 16, "f32", T=T, seed=sum(lengths)), 64)
