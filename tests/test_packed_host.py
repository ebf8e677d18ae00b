"""Packed batches without a GPU: what the calls refuse (before anything is launched), how large their memory is, and the 64-bit
reference of the GPU tests against differences and against itself."""
import ctypes
import os

import numpy as np
import pytest
import torch

import packed_ref as ref
from conftest import ROOT
from paper_2604_10597_amd import binding

P = ctypes.c_void_p(4096)           # stands for device memory: a refused call does not touch it
Q = ctypes.c_void_p(8192)
F32 = binding.COREY_F32


def index(S=3, T=100, tile=64, table=4096, size=None):
    size = binding.lib().corey_pack_bytes(S, T, tile) if size is None else size
    return binding.Pack(table, size, S, T, tile, 0)


def plan(lengths=P, S=3, T=100, tile=64, table=Q, size=1 << 20, pack=None):
    p = binding.Pack() if pack is None else pack
    return binding.lib().corey_pack_plan(lengths, S, T, tile, table, size, None if pack == 0 else ctypes.byref(p), None)


def conv(x=P, xs=8, w=P, state=P, n_slots=4, slots=None, out=None, pack=None, u=Q, us=8, dt=F32, D=8, W=4):
    pk = index() if pack is None else pack
    return binding.lib().corey_conv_packed(x, xs, w, None, state, n_slots, slots, out, None if pk == 0 else ctypes.byref(pk), u, us, dt, D, W, None)


def conv_bwd(x=P, xs=8, w=P, du=P, dus=8, pack=None, dx=Q, dxs=8, dw=P, dt=F32, D=8, W=4, ws=P, size=1 << 20):
    pk = index() if pack is None else pack
    return binding.lib().corey_conv_packed_bwd(x, xs, w, None, du, dus, ctypes.byref(pk), dx, dxs, dw, None, dt, D, W, ws, size, None)


def scan(u=P, us=8, A=P, bs=16, z=P, zs=8, state=None, n_slots=0, slots=None, pack=None, y=Q, ys=8, dt=F32, D=8, N=16, ws=P, size=1 << 22):
    pk = index() if pack is None else pack
    return binding.lib().corey_scan_packed(u, us, P, 8, A, P, bs, P, 16 if N <= 16 else N, None, z, zs, None, 1, state, n_slots, slots, None,
                                           ctypes.byref(pk), y, ys, dt, D, N, ws, size, None)


def step(state=P, n_slots=4, slots=P, x=P, xs=8, bs=16, y=Q, dt=F32, S=3, D=8, N=16):
    return binding.lib().corey_scan_packed_step(state, n_slots, slots, None, x, xs, P, xs, P, P, bs, P, bs, None, None, 0, None, 1, y, xs, dt, S, D, N, None)


def scan_bwd(u=P, z=P, dz=ctypes.c_void_p(1 << 16), du=ctypes.c_void_p(1 << 17), dd=ctypes.c_void_p(1 << 18), dB=ctypes.c_void_p(1 << 19),
             dC=ctypes.c_void_p(1 << 20), dA=P, pack=None, dt=F32, D=8, N=16, ws=P, size=1 << 24, stride=None):
    pk = index() if pack is None else pack
    n = N
    s = stride or D
    return binding.lib().corey_scan_packed_bwd(u, s, P, s, P, P, n, P, n, None, z, s, None, 1, P, s, ctypes.byref(pk), du, s, dd, s, dA, dB, n,
                                               dC, n, None, dz, s, None, dt, D, N, ws, size, None)


E = {v: k for k, v in binding.STATUS.items()}


@pytest.mark.parametrize("call, kw, code", [
    (plan, dict(lengths=None), "COREY_ENULL"), (plan, dict(table=None), "COREY_ENULL"), (plan, dict(pack=0), "COREY_ENULL"),
    (plan, dict(S=0), "COREY_ESHAPE"), (plan, dict(S=(1 << 20) + 1), "COREY_ESHAPE"), (plan, dict(T=0), "COREY_ESHAPE"),
    (plan, dict(T=1 << 31), "COREY_ESHAPE"), (plan, dict(tile=8), "COREY_EINVAL"), (plan, dict(tile=40), "COREY_EINVAL"),
    (plan, dict(tile=4096), "COREY_EINVAL"), (plan, dict(size=64), "COREY_EWORKSPACE"), (plan, dict(table=ctypes.c_void_p(8200)), "COREY_EWORKSPACE"),
    (conv, dict(x=None), "COREY_ENULL"), (conv, dict(w=None), "COREY_ENULL"), (conv, dict(u=None), "COREY_ENULL"), (conv, dict(u=P), "COREY_EINVAL"),
    (conv, dict(pack=0), "COREY_ENULL"), (conv, dict(pack=index(table=0)), "COREY_ENULL"), (conv, dict(pack=binding.Pack(4096, 100, 0, 1, 64, 0)), "COREY_EINVAL"),
    (conv, dict(pack=index(size=64)), "COREY_EWORKSPACE"), (conv, dict(pack=index(table=4100)), "COREY_EWORKSPACE"),
    (conv, dict(pack=binding.Pack(4096, 1 << 20, 3, 100, 40, 0)), "COREY_EINVAL"), (conv, dict(dt=7), "COREY_EINVAL"),
    (conv, dict(W=0), "COREY_EINVAL"), (conv, dict(W=5), "COREY_EINVAL"), (conv, dict(D=0), "COREY_ESHAPE"), (conv, dict(D=(1 << 20) + 1), "COREY_ESHAPE"),
    (conv, dict(xs=7), "COREY_ESHAPE"), (conv, dict(us=0), "COREY_ESHAPE"), (conv, dict(us=1 << 25), "COREY_ESHAPE"),
    (conv, dict(slots=P, state=None), "COREY_ENULL"), (conv, dict(out=P, n_slots=0), "COREY_ENULL"),
    (conv_bwd, dict(du=None), "COREY_ENULL"), (conv_bwd, dict(dx=None), "COREY_ENULL"), (conv_bwd, dict(dw=None), "COREY_ENULL"),
    (conv_bwd, dict(dx=P), "COREY_EINVAL"), (conv_bwd, dict(dus=3), "COREY_ESHAPE"), (conv_bwd, dict(ws=None), "COREY_EWORKSPACE"),
    (conv_bwd, dict(size=8), "COREY_EWORKSPACE"), (conv_bwd, dict(ws=ctypes.c_void_p(4098)), "COREY_EWORKSPACE"),
    (scan, dict(u=None), "COREY_ENULL"), (scan, dict(A=None), "COREY_ENULL"), (scan, dict(y=None), "COREY_ENULL"), (scan, dict(y=P), "COREY_EINVAL"),
    (scan, dict(dt=-1), "COREY_EINVAL"), (scan, dict(N=0), "COREY_ESHAPE"), (scan, dict(N=129, bs=129), "COREY_EUNSUPPORTED"), (scan, dict(bs=15), "COREY_ESHAPE"),
    (scan, dict(us=1), "COREY_ESHAPE"), (scan, dict(zs=1), "COREY_ESHAPE"), (scan, dict(ys=1), "COREY_ESHAPE"), (scan, dict(slots=P), "COREY_ENULL"),
    (scan, dict(ws=None), "COREY_EWORKSPACE"), (scan, dict(size=100), "COREY_EWORKSPACE"), (scan, dict(ws=ctypes.c_void_p(4100)), "COREY_EWORKSPACE"),
    (scan, dict(pack=binding.Pack(4096, 1 << 40, 1 << 20, (1 << 31) - 1, 16, 0), D=1 << 20, us=1 << 20, zs=1 << 20, ys=1 << 20), "COREY_ESHAPE"),
    (step, dict(state=None), "COREY_ENULL"), (step, dict(slots=None), "COREY_ENULL"), (step, dict(y=P), "COREY_EINVAL"), (step, dict(S=0), "COREY_ESHAPE"),
    (step, dict(N=257, bs=257), "COREY_ESHAPE"), (step, dict(S=1 << 20, D=64, xs=64), "COREY_ESHAPE"), (step, dict(bs=3), "COREY_ESHAPE"), (step, dict(dt=9), "COREY_EINVAL"),
    (step, dict(state=ctypes.c_void_p(4098)), "COREY_EINVAL"), (step, dict(n_slots=0), "COREY_ESHAPE"),
    (scan_bwd, dict(u=None), "COREY_ENULL"), (scan_bwd, dict(du=None), "COREY_ENULL"), (scan_bwd, dict(dA=None), "COREY_ENULL"), (scan_bwd, dict(dz=None), "COREY_ENULL"),
    (scan_bwd, dict(z=None), "COREY_ENULL"), (scan_bwd, dict(du=P), "COREY_EINVAL"), (scan_bwd, dict(dd=ctypes.c_void_p(1 << 17)), "COREY_EINVAL"),
    (scan_bwd, dict(N=129), "COREY_EUNSUPPORTED"), (scan_bwd, dict(pack=index(tile=128)), "COREY_EUNSUPPORTED"), (scan_bwd, dict(N=65), "COREY_EUNSUPPORTED"),
    (scan_bwd, dict(size=4), "COREY_EWORKSPACE"), (scan_bwd, dict(ws=None), "COREY_EWORKSPACE"), (scan_bwd, dict(dt=3), "COREY_EINVAL"), (scan_bwd, dict(stride=7), "COREY_ESHAPE"),
])
def test_refusals(call, kw, code):
    assert binding.STATUS[call(**kw)] == code
    assert binding.lib().corey_last_error()


def test_a_refused_plan_leaves_the_index_as_it_was():
    p = index()
    before = bytes(p)
    assert plan(pack=p, tile=5) != 0 and bytes(p) == before


def test_sizes():
    L = binding.lib()
    p = index(S=3, T=100, tile=64)
    up = lambda n: -(-n // 4) * 4
    words = 16 + up(4) + up(100) + 4 * (100 // 64 + 3) + 4 * (100 // 16 + 3) + 2 * up(4) + up(100 // 65)
    assert L.corey_pack_bytes(3, 100, 64) == 4 * words
    for bad in ((0, 1, 16), (1, 0, 16), (1, 1, 15), (1, 1, 4096), (1 << 21, 1, 16), (1, 1 << 31, 16)):
        assert L.corey_pack_bytes(*bad) == 0
    # B and C as binary32 by blocks of 16 tokens, and the tiles' states where a sequence can have a second tile
    relaid = lambda T: 4 * ((T // 16 + 3) * 16 * 32 + 48)
    assert L.corey_scan_packed_workspace(ctypes.byref(p), 8, 16) == relaid(100) + 4 * (100 // 64 + 3) * 17 * 8
    assert L.corey_scan_packed_workspace(ctypes.byref(index(T=64)), 8, 16) == relaid(64)
    assert L.corey_scan_packed_workspace(ctypes.byref(p), 8, 129) == 0 and L.corey_scan_packed_bwd_workspace(ctypes.byref(p), 0, 16) == 0
    assert L.corey_conv_packed_bwd_workspace(ctypes.byref(p), 8, 5) == 0 and L.corey_conv_packed_bwd_workspace(None, 8, 4) == 0


def test_tile_rule():
    t = binding.corey_pack_tile
    for S in (1, 7, 4000):
        for T in (1, 500, 16384, 1 << 20):
            for D in (1, 64, 2048, 5120):
                for N in (1, 16, 128):
                    tile = t(S, T, D, N)
                    assert 16 <= tile <= 2048 and tile % 16 == 0
                    back = t(S, T, D, N, backward=True)
                    assert back in (16, 32, 48, 64) and back <= (32 if N > 64 else 64)
    assert t(0, 1, 1, 1) == 0 and t(1, 1, 1, 0) == 0
    assert t(1, 1 << 20, 5120) >= t(1, 1 << 14, 5120) >= t(1, 1 << 10, 5120)
    assert 4096 <= -(-16384 // t(1, 16384, 5120)) * 80 <= 5120   # all tiles run at once


def test_parts_of_the_index_are_where_the_header_says():
    p = index(S=6, T=50, tile=16)
    table = torch.arange(p.bytes // 4 + 5, dtype=torch.int32)[5:]
    p.table, p._table = table, table.data_ptr()
    at = lambda part: (tuple(part.shape), part.stride(), (part.data_ptr() - table.data_ptr()) // 4)
    assert at(p.starts) == ((7,), (1,), 16) and at(p.seq) == ((50,), (1,), 24)
    assert at(p.tiles) == ((50 // 16 + 6, 4), (4, 1), 76) and at(p.blocks) == ((50 // 16 + 6, 4), (4, 1), 76 + 36)
    p.table = table[1:]                                           # another table than the index was built in
    with pytest.raises(ValueError):
        p.starts


# ------------------------------------------------------------------------------------------- the reference
def test_reference_plan_on_a_hand_written_batch():
    starts, seq, tiles, blocks = ref.plan([20, 0, -3, 2], 24, 32)
    assert starts.tolist() == [0, 20, 20, 20, 22] and seq.tolist() == [0] * 20 + [3, 3, -1, -1]
    assert tiles.tolist() == [[0, 0, 20, 3], [3, 20, 2, 3], [-1, 0, 0, 0], [-1, 0, 0, 0]]
    assert blocks.tolist()[:3] == [[0, 0, 16, 1], [0, 16, 4, 2], [3, 20, 2, 3]] and len(blocks) == 1 + 4
    assert ref.plan([5, 5], 7, 16)[0].tolist() == [0, 5, 7]


def rng_scan(n=7, D=3, N=2, seed=0, gated=True):
    g = np.random.default_rng(seed)
    return dict(u=g.standard_normal((n, D)), delta=g.standard_normal((n, D)), A=-np.exp(g.standard_normal((D, N))), B=g.standard_normal((n, N)),
                C=g.standard_normal((n, N)), Dv=g.standard_normal(D), z=g.standard_normal((n, D)) if gated else None, bias=g.standard_normal(D))


@pytest.mark.parametrize("gated, softplus", [(True, True), (False, True), (True, False)])
def test_reference_gradients_of_the_scan_against_differences(gated, softplus):
    v = rng_scan(gated=gated)
    if not softplus:
        v["delta"], v["bias"] = np.abs(v["delta"]), np.abs(v["bias"])
    dy = np.random.default_rng(9).standard_normal(v["u"].shape)
    out = lambda w: (ref.Scan(**w, softplus=softplus, h0=np.zeros(v["A"].shape), tile=16).forward("f32")[0] * dy).sum()
    grads = ref.Scan(**v, softplus=softplus, h0=np.zeros(v["A"].shape), tile=16).backward(dy, 4, 4)
    names = dict(u="du", delta="ddelta", A="dA", B="dB", C="dC", Dv="dD", z="dz", bias="ddelta_bias")
    for k, name in names.items():
        if v[k] is None:
            continue
        num = np.zeros_like(v[k])
        for i in np.ndindex(v[k].shape):
            w = {a: (b.copy() if b is not None else None) for a, b in v.items()}
            w[k][i] += 1e-6
            up = out(w)
            w[k][i] -= 2e-6
            num[i] = (up - out(w)) / 2e-6
        # central differences: truncation 1e-12 of the third derivative, cancellation 1e-16 / 1e-6 of the value
        assert np.allclose(grads[name][0], num, rtol=1e-7, atol=1e-7), name


def test_reference_gradients_of_the_convolution_against_differences():
    g = np.random.default_rng(1)
    for n, W in ((6, 4), (2, 4), (5, 1), (3, 2)):
        x, w, b, du = g.standard_normal((n, 2)), g.standard_normal((2, W)), g.standard_normal(2), g.standard_normal((n, 2))
        zero = np.zeros((2, W - 1))
        out = lambda x, w, b: (ref.conv(x, w, b, zero, "f32")[0] * du).sum()
        grads = ref.conv_bwd(x, w, b, du, "f32")
        for a, (got, _) in zip((x, w, b), grads):
            num = np.zeros_like(a)
            for i in np.ndindex(a.shape):
                old = a[i]
                a[i] = old + 1e-6
                up = out(x, w, b)
                a[i] = old - 1e-6
                num[i] = (up - out(x, w, b)) / 2e-6
                a[i] = old
            assert np.allclose(got, num, rtol=1e-7, atol=1e-7)


def test_reference_scan_continues_where_it_stopped():
    v = rng_scan(n=12, seed=3)
    part = lambda f, e, h0: ref.Scan(*[v[k][f:e] if k in ("u", "delta", "B", "C", "z") else v[k] for k in ("u", "delta", "A", "B", "C", "Dv", "z", "bias")],
                                     softplus=True, h0=h0, tile=16)
    whole = part(0, 12, np.zeros((3, 2)))
    a = part(0, 5, np.zeros((3, 2)))
    b = part(5, 12, a.last()[0])
    assert np.allclose(np.concatenate([a.forward("f32")[0], b.forward("f32")[0]]), whole.forward("f32")[0], rtol=1e-14, atol=1e-14)
    assert np.allclose(b.last()[0], whole.last()[0], rtol=1e-14, atol=1e-14)


def test_reference_agrees_with_the_c_oracle():
    import oracle
    v = rng_scan(n=20, D=4, N=3, seed=5)
    t = lambda a: np.ascontiguousarray(a.T[None], np.float32)
    f = lambda a: np.ascontiguousarray(a, np.float32)
    v = {k: f(a).astype(np.float64) for k, a in v.items()}
    st, y, last = oracle.selective_scan(t(v["u"]), t(v["delta"]), f(v["A"]), t(v["B"]), t(v["C"]), Dv=f(v["Dv"]), z=t(v["z"]), delta_bias=f(v["bias"]))
    r = ref.Scan(**v, softplus=True, h0=np.zeros((4, 3)), tile=16)
    assert st == 0 and np.allclose(y[0].T, r.forward("f32")[0], rtol=1e-12, atol=1e-12) and np.allclose(last[0], r.last()[0], rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("mistake", ["state", "gate", "skip", "decay"])
def test_the_bounds_notice_a_mistake_of_a_thousandth(mistake):
    """The reference's own bounds, on a reference with one factor off by 1e-3 (the mistakes are planted here, on the CPU)."""
    v = rng_scan(n=40, D=8, N=16, seed=7)
    h0 = np.random.default_rng(2).standard_normal((8, 16))
    make = lambda w, h: ref.Scan(**w, softplus=True, h0=h, tile=64)
    y, bound = make(v, h0).forward("f32")
    w, h = dict(v), h0
    if mistake == "state":
        h = h0 * 1.001
    elif mistake == "gate":
        w["z"] = v["z"] * 1.001
    elif mistake == "skip":
        w["Dv"] = v["Dv"] * 1.001
    else:
        w["A"] = v["A"] * 1.001
    with pytest.raises(AssertionError):
        ref.check(make(w, h).forward("f32")[0], y, bound, mistake)


def test_the_binding_knows_every_entry_point():
    hdr = open(os.path.join(ROOT, "include", "corey.h")).read()
    for name in ("corey_pack_plan", "corey_conv_packed", "corey_scan_packed", "corey_scan_packed_step", "corey_scan_packed_bwd", "corey_conv_packed_bwd"):
        assert f"int {name}(" in hdr and name in binding.EXPORTS and callable(getattr(binding, name))
