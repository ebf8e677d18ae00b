"""Packed batches on streams: every call is ordered behind the work of the stream it is made on."""
import pytest
import torch

import paper_2604_10597_amd as corey
from packed_util import Batch

pytestmark = pytest.mark.gpu

DEV = "cuda"


class Layer:
    """A batch through every operator: index, convolution, scan, both gradients, and one token more of every sequence."""

    def __init__(self, seed):
        self.b = b = Batch([300, 40, 5], 256, 16, "bf16", seed=seed)
        g = torch.Generator(device=DEV).manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, device=DEV, generator=g).bfloat16()
        self.w = torch.randn(256, 4, device=DEV, generator=g) / 2
        self.inputs = dict(lens=b.lens(), slots=torch.tensor([2, 0, 1], dtype=torch.int32, device=DEV), x=rnd(b.T, 256), delta=b.delta, B=b.B, C=b.C,
                           z=b.z, dy=b.dy, x1=rnd(3, 256), delta1=rnd(3, 256), B1=rnd(3, 16), C1=rnd(3, 16),
                           conv_pool=rnd(3, 256, 3), pool=torch.randn(3, 256, 16, device=DEV, generator=g))

    def run(self):
        b, i = self.b, self.inputs
        kw = dict(Dv=b.Dv, delta_bias=b.bias)
        pack = corey.corey_pack_plan(i["lens"], b.T, 48)
        u = corey.corey_conv_packed(i["x"], self.w, None, pack, state=i["conv_pool"], slots=i["slots"])
        y = corey.corey_scan_packed(u, i["delta"], b.A, i["B"], i["C"], pack, z=i["z"], state=i["pool"], slots=i["slots"], **kw)
        y1 = corey.corey_scan_packed_step(i["pool"], i["slots"], i["x1"], i["delta1"], b.A, i["B1"], i["C1"], **kw)
        g = corey.corey_scan_packed_bwd(u, i["delta"], b.A, i["B"], i["C"], pack, i["dy"], z=i["z"], **kw)
        return [pack.starts, pack.seq, u, y, y1, *(g[k] for k in sorted(g)), *corey.corey_conv_packed_bwd(i["x"], self.w, None, g["du"], pack),
                i["conv_pool"], i["pool"]]


@pytest.mark.parametrize("streams", [1, 2])
def test_calls_wait_for_their_streams_work(streams):
    """The inputs hold other values until work of the stream's own, which is still under way when the calls are made, puts the right ones
    there: a call that went ahead of it would give other results."""
    layers = [Layer(s) for s in range(streams)]
    right = [{k: v.clone() for k, v in x.inputs.items()} for x in layers]
    want = [[t.clone() for t in x.run()] for x in layers]
    for x in layers:
        for k, v in x.inputs.items():
            v.fill_(1 if v.dtype == torch.int32 else 7)          # (lengths and slots that are valid, too)
        x.inputs["slots"].copy_(torch.tensor([0, 1, 2], dtype=torch.int32))
    big = torch.randn(4096, 4096, device=DEV) / 64
    torch.cuda.synchronize()
    got, busy = [], []
    for x, values in zip(layers, right):
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            late = big
            for _ in range(60):
                late = late @ big
            at = torch.cuda.Event()
            at.record()
            for k, v in x.inputs.items():
                v.copy_(values[k])
            got.append(x.run())
            busy.append(at)
    assert not any(at.query() for at in busy), "the calls were made behind finished work: nothing was tested"
    torch.cuda.synchronize()
    for a, c in zip(want, got):
        for p, q in zip(a, c):
            assert torch.equal(p, q)
