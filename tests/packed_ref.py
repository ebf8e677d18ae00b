"""The operators on packed batches in 64 bits (numpy, sequence by sequence and token by token), each with a bound on what binary32
arithmetic may be off: every rounding is followed through the recurrences in absolute values.

Let r = 2^-24, half a step of binary32, relative.  Where the kernels round:
  raw = delta + bias: r |raw|, absolute.  softplus multiplies an absolute error of raw by at most its own derivative <= dl (small
      raw) or 1, i.e. relative to dl at most |raw| r; its own exponential, logarithm and sums add a few r.  dl is off by
      ETA = (3 |raw| + 8) r, relative.
  a = exp(dl A): the argument has two products and its scaling, each r, and dl's ETA; the exponential's own error is 2 r:
      relative |dl A| (3 r + ETA) + 2 r.  Over a tile the argument is A times a sum of step sizes, whose additions are off by
      (tokens of a tile) r relative at most: |dl A| tile r on top.
  b = dl u B: ETA + 2 r.   The update and every sum: r of the absolute values, once per addition on the way.
A sum over n values by any tree whose longest path has k additions is off by k r of the sum of the absolute values.
Storage: half a step of the type, eps / 2 of the value, and half the spacing of the smallest values below the normal range."""
from __future__ import annotations

import numpy as np

R = 2.0 ** -24
STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -24}     # (gfx950 flushes no binary16; binary32 may be flushed)


def stored(value, err, dtype):
    """The bound after the value is rounded to `dtype`."""
    return err + STEP[dtype] * (np.abs(value) + err) + TINY[dtype]


def check(got, ref, bound, what):
    got = np.asarray(got, np.float64)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert np.isfinite(got).all(), f"{what}: non-finite"
    bad = np.abs(got - ref) > bound
    if bad.any():
        i = np.unravel_index(np.argmax(np.abs(got - ref) / bound), got.shape)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} beyond their bound; worst at {i}: {got[i]!r}, expected {ref[i]!r}, bound {bound[i]:.3e}")


def spans(lengths, T):
    """[first, stop) of every sequence: negative lengths are 0, what does not fit into T rows is cut off."""
    out, at = [], 0
    for n in lengths:
        stop = min(T, at + max(0, int(n)))
        out.append((at, stop))
        at = stop
    return out


def plan(lengths, T, tile):
    sp = spans(lengths, T)
    starts = np.array([f for f, _ in sp] + [sp[-1][1]], np.int32)
    seq = np.full(T, -1, np.int32)
    for s, (f, e) in enumerate(sp):
        seq[f:e] = s
    tables = []
    for size in (tile, 16):
        rows = [[s, at, min(size, e - at), (at == f) + 2 * (at + size >= e)] for s, (f, e) in enumerate(sp) for at in range(f, e, size)]
        room = T // size + min(len(lengths), T)
        assert len(rows) <= room
        tables.append(np.array(rows + [[-1, 0, 0, 0]] * (room - len(rows)), np.int32).reshape(room, 4))
    return starts, seq, tables[0], tables[1]


def sigmoid(v):
    return np.exp(-np.logaddexp(0.0, -v))


def conv(x, w, b, state, dtype):
    """One sequence: x [n, D], w [D, W], state [D, W-1].  (u, its bound, the new state)."""
    W = w.shape[1]
    full = np.concatenate([state.T, x], 0) if W > 1 else x
    n = x.shape[0]
    v = np.broadcast_to(b, x.shape).copy()
    mag = np.abs(v)
    for k in range(W):
        v = v + w[:, k] * full[k:k + n]
        mag = mag + np.abs(w[:, k] * full[k:k + n])
    ev = W * R * mag
    sig = sigmoid(v)
    # |silu'| <= 1.1; the exponential's argument is off by |v| 2 r, the sigmoid by its own sum, reciprocal and exponential
    err = 1.1 * ev + np.abs(v) * sig * (2 * np.abs(v) + 6) * R
    u = v * sig
    return u, stored(u, err, dtype), full[n:].T if W > 1 else state


def conv_bwd(x, w, b, du, dtype, more=0):
    """One sequence from zero: (dx, bound), (dw, bound), (db, bound); `more`: additions over runs of pieces."""
    n, D = x.shape
    W = w.shape[1]
    full = np.concatenate([np.zeros((W - 1, D)), x], 0)
    v = np.broadcast_to(b, x.shape).copy()
    mag = np.abs(v)
    for k in range(W):
        v = v + w[:, k] * full[k:k + n]
        mag = mag + np.abs(w[:, k] * full[k:k + n])
    ev = W * R * mag
    sig = sigmoid(v)
    slope = sig * (1 + v * (1 - sig))
    # |silu''| <= 1/2; the slope's own roundings: sigmoid (2 |v| + 6) r, then two products and a sum of (1 + |v|)
    es = 0.5 * ev + (1 + np.abs(v)) * (2 * np.abs(v) + 10) * R
    dv = du * slope
    ed = np.abs(du) * es + R * np.abs(dv)
    dx, ex = np.zeros_like(x), np.zeros_like(x)
    for k in range(W):
        a = W - 1 - k
        if a < n:
            dx[:n - a] += w[:, k] * dv[a:]
            ex[:n - a] += np.abs(w[:, k]) * (ed[a:] + W * R * np.abs(dv[a:]))
    dw = np.stack([(dv * full[k:k + n]).sum(0) for k in range(W)], 1)
    depth = n + more + 8
    ew = np.stack([((ed + depth * R * np.abs(dv)) * np.abs(full[k:k + n])).sum(0) for k in range(W)], 1)
    return (dx, stored(dx, ex, dtype)), (dw, ew + TINY["f32"]), (dv.sum(0), (ed + depth * R * np.abs(dv)).sum(0) + TINY["f32"])


class Scan:
    """One sequence through the scan, forward and backward, from state h0 [D, N] (the backward pass wants zeros)."""

    def __init__(self, u, delta, A, B, C, Dv, z, bias, softplus, h0, tile):
        n, D = u.shape
        N = A.shape[1]
        self.u, self.A, self.B, self.C, self.Dv, self.z, self.n, self.tile = u, A, B, C, Dv, z, n, tile
        self.raw = delta + bias
        self.softplus = softplus
        self.dl = np.logaddexp(0.0, self.raw) if softplus else self.raw
        self.eta = (3 * np.abs(self.raw) + 8) * R if softplus else np.full_like(self.raw, 2 * R)
        x = self.dl[:, :, None] * A                                   # [n, D, N]
        self.a = np.exp(x)
        self.ea = np.abs(x) * ((3 + tile) * R + self.eta[:, :, None]) + 2 * R
        self.dx = self.dl * u
        b = self.dx[:, :, None] * B[:, None]
        eb = np.abs(b) * (self.eta[:, :, None] + 3 * R)
        self.h, self.eh = np.empty((n + 1, D, N)), np.empty((n + 1, D, N))
        self.h[0], self.eh[0] = h0, 0.0
        H = np.abs(h0)
        for t in range(n):
            self.h[t + 1] = self.a[t] * self.h[t] + b[t]
            kept = self.a[t] * H
            H = kept + np.abs(b[t])
            self.eh[t + 1] = self.a[t] * self.eh[t] + kept * self.ea[t] + eb[t] + 3 * R * H
        skip = Dv * u
        read = np.abs(C[:, None] * self.h[1:])
        self.s = (self.h[1:] * C[:, None]).sum(-1) + skip
        self.es = (np.abs(C[:, None]) * self.eh[1:] + (N + 2) * R * read).sum(-1) + (N + 2) * R * np.abs(skip)
        if z is None:
            self.gate, self.eg = np.ones_like(u), np.zeros_like(u)
        else:
            self.sig = sigmoid(z)
            self.gate = z * self.sig
            self.eg = np.abs(self.gate) * (2 * np.abs(z) + 6) * R

    def forward(self, dtype):
        y = self.s * self.gate
        return y, stored(y, self.es * np.abs(self.gate) + np.abs(self.s) * self.eg + R * np.abs(y), dtype)

    def last(self):
        return self.h[-1], self.eh[-1] + R * np.abs(self.h[-1]) + TINY["f32"]

    def backward(self, dy, channel_adds, tile_adds):
        """name -> (value, bound before the storage's rounding); the sums over channels and over tiles take that many additions."""
        n, D = dy.shape
        N = self.A.shape[1]
        ds = dy * self.gate
        eds = np.abs(dy) * self.eg + R * np.abs(ds)
        g, eg = np.empty_like(self.a), np.empty_like(self.a)
        now, enow, G = np.zeros((D, N)), np.zeros((D, N)), np.zeros((D, N))
        absg = np.empty_like(self.a)
        for t in range(n - 1, -1, -1):
            term = ds[t][:, None] * self.C[t]
            now = now + term
            G = G + np.abs(term)
            enow = enow + eds[t][:, None] * np.abs(self.C[t]) + 3 * R * G
            g[t], eg[t], absg[t] = now, enow, G
            enow = self.a[t] * enow + self.a[t] * G * (self.ea[t] + 2 * R)
            now, G = self.a[t] * now, self.a[t] * G
        kept = self.a * self.h[:-1]
        ekept = self.a * self.eh[:-1] + np.abs(kept) * (self.ea + 2 * R)
        out = {}
        out["dC"] = ((ds[:, :, None] * self.h[1:]).sum(1),
                     (np.abs(ds)[:, :, None] * self.eh[1:] + eds[:, :, None] * np.abs(self.h[1:]) + (channel_adds + 2) * R * np.abs(ds[:, :, None] * self.h[1:])).sum(1))
        dx, edx = self.dx[:, :, None], np.abs(self.dx)[:, :, None] * (self.eta[:, :, None] + 2 * R)
        out["dB"] = ((g * dx).sum(1), (eg * np.abs(dx) + np.abs(g) * edx + (channel_adds + 2) * R * np.abs(g * dx)).sum(1))
        gb = (g * self.B[:, None]).sum(-1)
        egb = (eg * np.abs(self.B[:, None]) + (N + 2) * R * np.abs(g * self.B[:, None])).sum(-1)
        out["du"] = (self.Dv * ds + self.dl * gb, np.abs(self.Dv) * eds + np.abs(self.dl) * (egb + (self.eta + 3 * R) * np.abs(gb)) + 3 * R * np.abs(self.Dv * ds))
        through = g * kept
        et = eg * np.abs(kept) + np.abs(g) * ekept + eg * ekept + 2 * R * np.abs(through)
        ga = (through * self.A).sum(-1)
        ega = ((et + (N + 5) * R * np.abs(through)) * np.abs(self.A)).sum(-1)
        ddl = gb * self.u + ga
        eddl = egb * np.abs(self.u) + ega + 3 * R * (np.abs(gb * self.u) + np.abs(ga))
        if self.softplus:
            sg = sigmoid(self.raw)
            eddl = eddl * sg + np.abs(ddl) * sg * (3 * np.abs(self.raw) + 8) * R
            ddl = ddl * sg
        out["ddelta"] = (ddl, eddl)
        depth = self.tile + tile_adds + 8
        out["ddelta_bias"] = (ddl.sum(0), (eddl + depth * R * np.abs(ddl)).sum(0))
        dl = self.dl[:, :, None]
        out["dA"] = ((through * dl).sum(0), ((et + (self.eta[:, :, None] + depth * R) * np.abs(through)) * np.abs(dl)).sum(0))
        out["dD"] = ((ds * self.u).sum(0), ((eds + depth * R * np.abs(ds)) * np.abs(self.u)).sum(0))
        if self.z is not None:
            slope = self.sig * (1 + self.z * (1 - self.sig))
            esl = (1 + np.abs(self.z)) * (2 * np.abs(self.z) + 10) * R
            out["dz"] = (dy * self.s * slope, np.abs(dy) * (self.es * np.abs(slope) + np.abs(self.s) * esl + 3 * R * np.abs(self.s * slope)))
        return out
