"""Packed batches at the edges of their numbers: decays that overflow beside zeros."""
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
