"""Packed batches large enough for what small ones never reach: two sets of rows a workgroup in the single-token scan, several pieces a
run in the convolution's gradients."""
import numpy as np
import pytest
import torch

import packed_ref as ref
import paper_2604_10597_amd as corey
from packed_util import Batch, f64, rows
from paper_2604_10597_amd import binding

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(np.asarray(v, np.int32)).cuda()


# ------------------------------------------------------------------------------------------- single tokens, two sets a workgroup
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("dtype, S, D, N, lay, gated", [
    ("bf16", 41, 2201, 16, "wide", True),            # 1411 sets, the last of them with four rows' lanes
    ("f32", 34, 2650, 16, "plain", False),           # 1408
    ("f16", 30, 3001, 12, "odd", True),              # 1407; a row of three groups on four lanes
    ("f32", 13, 3461, 20, "odd", True)])             # 1407; of five on eight
def test_many_single_tokens(dtype, S, D, N, lay, gated, in_place):
    lanes = 1 << (-(-N // 4) - 1).bit_length()
    assert -(-S * D * lanes // 256) > 1400
    b = Batch([1] * S, D, N, dtype, seed=S + N, lay=lay, gated=gated, skip=gated, bias=gated)
    g = np.random.default_rng(2)
    pool64 = g.standard_normal((2 * S + 1, D, N)).astype(np.float32)
    pool = torch.from_numpy(pool64).cuda()
    order = g.permutation(2 * S + 1)
    read = order[:S].copy()
    read[1] = -1                                     # begins from zero; in place it is not kept
    write = read if in_place else order[S:2 * S].copy()
    if not in_place:
        write[2] = 2 * S + 1                         # not kept
    y = torch.full((S + 1, D), 9.0, dtype=b.u.dtype, device="cuda")
    corey.corey_scan_packed_step(pool, ints(read), b.u, b.delta, b.A, b.B, b.C, Dv=b.Dv, z=b.z, delta_bias=b.bias,
                                 slots_out=None if in_place else ints(write), y=y[:S])
    got = pool.cpu().numpy()
    kept = set()
    for s in range(S):
        r = b.scan(s, pool64[read[s]].astype(np.float64) if read[s] >= 0 else None, True, 1)
        ref.check(f64(y[s:s + 1]), *r.forward(dtype), f"y of {s}")
        if 0 <= write[s] <= 2 * S:
            kept.add(int(write[s]))
            ref.check(got[write[s]], *r.last(), f"state of {s}")
    for k in range(2 * S + 1):
        if k not in kept:
            assert np.array_equal(got[k], pool64[k]), f"slot {k} was not to be written"
    assert (y[S:] == 9.0).all()


# ------------------------------------------------------------------------------------------- the convolution's gradients, several pieces a run
SPREAD = [0, 1, 2, 3, 15, 16, 17, 0, 700, 5, 1, 1, 64, 33, 400, 2, 31, 48, 3, 600, 1, 0, 18, 2]


@pytest.mark.parametrize("dtype, D, W, lay, bias, lengths", [
    ("bf16", 8192, 4, "plain", True, SPREAD), ("f32", 4097, 4, "odd", True, SPREAD), ("f16", 4098, 3, "wide", True, SPREAD),
    ("f32", 8192, 2, "plain", False, SPREAD), ("bf16", 4097, 1, "plain", True, SPREAD), ("f32", 8191, 4, "plain", True, [1] * 300 + [2] * 100 + [3] * 100 + [1000]),
    ("bf16", 8192, 4, "wide", True, [3000])])
def test_gradients_of_the_convolution_over_runs_of_pieces(dtype, D, W, lay, bias, lengths):
    """Runs that carry on from piece to piece, through the ends of sequences, that end inside one, and a last one that is not full.  Every
    sequence's dx, and dweight and dbias over all, of the first and last channels of a launch's groups."""
    used, T = sum(lengths), sum(lengths) + 11
    g = np.random.default_rng(D + W)
    some = np.unique(np.r_[0:70, D // 2:D // 2 + 66, D - 70:D])
    x64, du64 = np.zeros((T, some.size)), np.zeros((T, some.size))
    x, xa = rows(g.standard_normal((T, D), np.float32), dtype, lay)
    du, dua = rows(g.standard_normal((T, D), np.float32), dtype, lay)
    x64, du64 = xa[:, some], dua[:, some]
    w = (g.uniform(-1, 1, (D, W)) / W ** 0.5).astype(np.float32)
    b = (g.uniform(-1, 1, D) / W ** 0.5).astype(np.float32)
    pack = corey.corey_pack_plan(ints(lengths), T, 64)
    runs = binding.lib().corey_conv_packed_bwd_workspace(pack, D, W) // (4 * (W + 1) * D)
    pieces = len(ref.plan(lengths, T, 64)[3])
    run = -(-pieces // runs)
    assert run > 1
    dx, dw, db = corey.corey_conv_packed_bwd(x, torch.from_numpy(w).cuda(), torch.from_numpy(b).cuda() if bias else None, du, pack)
    again = corey.corey_conv_packed_bwd(x, torch.from_numpy(w).cuda(), torch.from_numpy(b).cuda() if bias else None, du, pack)
    assert torch.equal(dx[:used], again[0][:used]) and torch.equal(dw, again[1]) and torch.equal(db, again[2]), "the order of the sums is fixed"
    w64, b64 = w[some].astype(np.float64), b[some].astype(np.float64) * bias
    got = f64(dx[:used])[:, some]
    sums = [0.0, 0.0, 0.0, 0.0]
    for s, (f, e) in enumerate(ref.spans(lengths, T)):
        if e == f:
            continue
        # a value is added to at most 16 tokens of each piece of its run, then the runs are
        (rx, bx), rw, rb = ref.conv_bwd(x64[f:e], w64, b64, du64[f:e], dtype, more=16 * run + runs)
        ref.check(got[f:e], rx, bx, f"dx of sequence {s}")
        sums = [a + v for a, v in zip(sums, (*rw, *rb))]
    ref.check(f64(dw)[some], sums[0], sums[1], "dweight")
    ref.check(f64(db)[some], sums[2], sums[3], "dbias")
