"""Packed batches at the edges: decays that overflow beside zeros, decays of 0, tables that are mostly empty."""
import numpy as np
import pytest
import torch

import packed_ref as ref
import paper_2604_10597_amd as corey
from packed_util import Batch, f64, rounded

pytestmark = pytest.mark.gpu

DEV = "cuda"


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------- growing states
@pytest.mark.parametrize("N", [4, 20])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_growing_states_from_zero_behind_a_tile(dtype, N):
    """Step sizes below 0 (no softplus) over the first block of a sequence's second tile: the decays there multiply to more than binary32
    holds, but the state that comes to them is 0 (B is until then) and so is the gradient (dy is 0 behind them): finite forward, so
    finite backward."""
    D, n, tile, at = 8, 128, 64, 64
    b = Batch([n], D, N, dtype, seed=3, gated=False, skip=False, bias=False)
    b.A64 = -np.ones((D, N))
    b.A = torch.from_numpy(b.A64.astype(np.float32)).to(DEV)
    delta = np.full((n, D), 0.125)
    delta[at:at + 16] = -5.625                                   # 16 decays of e^5.625: e^90 is beyond binary32's e^88.7
    bm, dy = b.B64.copy(), 1e-6 * b.dy64
    bm[:at + 16] = 0.0
    dy[at + 16:] = 0.0
    dy[at:at + 8] = 0.0                                          # (and half of them: what a step of 8 tokens hands back is 0 as well)
    b.delta, b.delta64 = (x.to(DEV) if torch.is_tensor(x) else x for x in rounded(delta, dtype))
    b.B, b.B64 = (x.to(DEV) if torch.is_tensor(x) else x for x in rounded(bm, dtype))
    b.dy, b.dy64 = (x.to(DEV) if torch.is_tensor(x) else x for x in rounded(dy, dtype))
    pack = corey.corey_pack_plan(b.lens(), n, tile)
    y = corey.corey_scan_packed(b.u, b.delta, b.A, b.B, b.C, pack, delta_softplus=False)
    r = b.scan(0, None, False, tile)
    ref.check(f64(y), *r.forward(dtype), "y")
    g = corey.corey_scan_packed_bwd(b.u, b.delta, b.A, b.B, b.C, pack, b.dy, delta_softplus=False)
    back = r.backward(b.dy64, 12, n // 16 + 1)
    for k in ("du", "ddelta", "dB", "dC"):
        ref.check(f64(g[k]), back[k][0], ref.stored(*back[k], dtype), k)
    ref.check(f64(g["dA"]), back["dA"][0], back["dA"][1] + ref.TINY["f32"], "dA")


# ------------------------------------------------------------------------------------------- decays of 0
@pytest.mark.parametrize("value", [-3e38, float("-inf")])
@pytest.mark.parametrize("N, tile", [(16, 16), (16, 64), (20, 32)])
def test_states_that_keep_nothing(N, tile, value):
    """Some of A so far below 0 that its product with log2(e) is no number of binary32 (or that it is none itself): those states hold the last
    token's product alone.  The tokens that fill up a sequence's last piece have a step size of 0 and change nothing."""
    lengths, D = [21, 1, 0, 70, 16, 9], 70
    b = Batch(lengths, D, N, "f32", seed=N + tile)
    gone = np.random.default_rng(1).random((D, N)) < 0.3
    b.A64 = np.where(gone, -1e8, b.A64)                          # the reference's: exp(-1e8 dl) is 0 in 64 bits for dl > 8e-6
    b.A = torch.from_numpy(np.where(gone, value, b.A64).astype(np.float32)).to(DEV)
    pack = corey.corey_pack_plan(b.lens(), b.T, tile)
    pool = torch.full((len(lengths), D, N), 9.0, device=DEV)
    kw = dict(Dv=b.Dv, z=b.z, delta_bias=b.bias)
    y = corey.corey_scan_packed(b.u, b.delta, b.A, b.B, b.C, pack, state=pool, slots=ints(*[-1] * 6), slots_out=ints(*range(6)), **kw)
    g = corey.corey_scan_packed_bwd(b.u, b.delta, b.A, b.B, b.C, pack, b.dy, **kw)
    sums = {}
    for s, (f, e) in enumerate(b.spans):
        if e == f:
            continue
        r = b.scan(s, None, True, tile)
        assert r.dl.min() > 8e-6
        ref.check(f64(y[f:e]), *r.forward("f32"), f"y of sequence {s}")
        ref.check(f64(pool[s]), *r.last(), f"state of sequence {s}")
        for k, (v, err) in r.backward(b.dy64[f:e], 12, b.T // 16 + 6).items():
            if k in ("dA", "dD", "ddelta_bias"):
                old = sums.get(k, (0.0, 0.0))
                sums[k] = (old[0] + v, old[1] + err)
            else:
                ref.check(f64(g[k][f:e]), v, ref.stored(v, err, "f32"), f"{k} of sequence {s}")
    for k, (v, err) in sums.items():
        ref.check(f64(g[k]), v, err + ref.TINY["f32"], k)


# ------------------------------------------------------------------------------------------- the index
@pytest.mark.parametrize("S", [3, 64, 4096, 4097, 131072])
def test_plan_of_a_table_that_is_mostly_empty(S):
    """A table of requests of which few have tokens: the empty entries between two of them are passed in one go, whatever their number."""
    inside = [5] + [0] * (S - 3) + [1, 7]
    behind = [5, 1, 7] + [0] * (S - 3)
    took = []
    for lengths in (inside, behind):
        lens, T = ints(*lengths), 15
        p = corey.corey_pack_plan(lens, T, 16)
        for got, want, what in zip((p.starts, p.seq, p.tiles, p.blocks), ref.plan(lengths, T, 16), ("starts", "seq", "tiles", "blocks")):
            assert np.array_equal(got.cpu().numpy(), want), what
        times = []
        for _ in range(5):
            first, last = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            first.record()
            corey.corey_pack_plan(lens, T, 16, table=p.table)
            last.record()
            torch.cuda.synchronize()
            times.append(first.elapsed_time(last))
        took.append(min(times))
    assert took[0] < 3 * took[1] + 0.05, took                    # ms; one by one 131072 of them take 9, of 0.3 for the sums
