"""Inputs of the packed-batch tests and the reference over all sequences of a batch."""
from __future__ import annotations

import numpy as np
import torch

import packed_ref as ref

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def rounded(a, dtype):
    """(torch tensor of the storage type, the values it holds in 64 bits)"""
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(TORCH[dtype])
    return t, t.to(torch.float64).numpy()


def rows(a, dtype, lay):
    """On the GPU as rows of the wanted layout: 'plain', 'wide' (the second half of longer rows), 'odd' (an odd row distance, from an odd
    element on)."""
    t, v = rounded(a, dtype)
    n, d = t.shape
    if lay == "plain":
        return t.cuda(), v
    big, at = (2 * d, d) if lay == "wide" else (d + 3 + d % 2, 1)
    whole = torch.full((n, big), float("nan"), dtype=t.dtype)
    whole[:, at:at + d] = t
    return whole.cuda()[:, at:at + d], v


class Batch:
    """A packed batch: `lengths` in T rows, everything the scan takes, seeded."""

    def __init__(self, lengths, D, N, dtype="f32", T=None, seed=0, lay="plain", gated=True, skip=True, bias=True):
        g = np.random.default_rng(seed)
        self.lengths, self.D, self.N, self.dtype = list(lengths), D, N, dtype
        total = sum(max(0, n) for n in self.lengths)
        self.T = T or max(1, total)
        self.spans = ref.spans(self.lengths, self.T)
        n = self.T
        self.u, self.u64 = rows(g.standard_normal((n, D)), dtype, lay)
        self.delta, self.delta64 = rows(0.5 * g.standard_normal((n, D)), dtype, lay)
        self.B, self.B64 = rows(g.standard_normal((n, N)), dtype, lay)
        self.C, self.C64 = rows(g.standard_normal((n, N)), dtype, lay)
        self.A64 = (-np.exp(0.5 * g.standard_normal((D, N))) * np.arange(1, N + 1) / 2).astype(np.float32).astype(np.float64)
        self.A = torch.from_numpy(self.A64.astype(np.float32)).cuda()
        self.z, self.z64 = rows(g.standard_normal((n, D)), dtype, lay) if gated else (None, None)
        self.Dv64 = g.standard_normal(D).astype(np.float32).astype(np.float64) if skip else np.zeros(D)
        self.Dv = torch.from_numpy(self.Dv64.astype(np.float32)).cuda() if skip else None
        self.bias64 = (np.log(1e-3) + g.random(D) * np.log(100.0)).astype(np.float32).astype(np.float64) if bias else np.zeros(D)
        self.bias = torch.from_numpy(self.bias64.astype(np.float32)).cuda() if bias else None
        self.dy, self.dy64 = rows(0.1 * g.standard_normal((n, D)), dtype, lay)

    def lens(self):
        return torch.tensor(self.lengths, dtype=torch.int32, device="cuda")

    def scan(self, s, h0=None, softplus=True, tile=64):
        f, e = self.spans[s]
        return ref.Scan(self.u64[f:e], self.delta64[f:e], self.A64, self.B64[f:e], self.C64[f:e], self.Dv64,
                        None if self.z64 is None else self.z64[f:e], self.bias64, softplus,
                        np.zeros((self.D, self.N)) if h0 is None else h0, tile)


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()
