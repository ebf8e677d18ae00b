"""The operators on packed batches, as cases to be timed and checked.

A packed batch holds the tokens of all its sequences one after another, [T, D], without padding; the states of the sequences
(the last inputs of the convolution, the state of the scan) lie in pools and are found by slot.  `kind` names the operator:

  plan       the index of a packed batch from the lengths of its sequences: where each begins, which token belongs to which,
             and the pieces of at most `tile` and of at most 16 tokens that the other operators work on
  conv       causal depthwise convolution and SiLU, begun from the slots' states, which move on
  conv_bwd   its gradients
  scan       the selective scan, begun from the slots' states, which move on
  step       the scan for one token of every sequence
  scan_bwd   the scan's gradients

`own` false: plain torch operations.  `own` true: the framework's calls on the same data.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
BLOCK = 16         # tokens of the small pieces
MOST = 84e6        # values of [T, D] in the largest listed case
STEPS = 16384      # tokens of the longest listed sequence


# ------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one generation step of a serving batch: 64 requests of one token or a few drafted ones
        dict(name="plan_tokens", kind="plan", S=64, T=120, spare=8, longest=5, tile=16),
        # a large packed training batch: 2000 documents in 256 K tokens, some of them empty
        dict(name="plan_documents", kind="plan", S=2000, T=262144, spare=0, longest=2048, tile=64),
        # the convolution of a generation step, 5120 channels, 64 requests
        dict(name="conv_tokens", kind="conv", dtype="bf16", S=64, T=64, spare=0, longest=1, D=5120, W=4, wide=True, carried=True),
        # prompts of many lengths through the convolution, 16384 tokens of 5120 channels; x is one half of the projection's rows
        dict(name="conv_prompts", kind="conv", dtype="bf16", S=24, T=16384, spare=0, longest=4096, D=5120, W=4, wide=True, carried=True),
        # the convolution's gradients in a small layer, binary32
        dict(name="conv_bwd_fp32", kind="conv_bwd", dtype="fp32", S=13, T=4099, spare=0, longest=1000, D=1536, W=4, wide=False),
        # ... and of a training batch of documents in a large one
        dict(name="conv_bwd_documents", kind="conv_bwd", dtype="bf16", S=19, T=16384, spare=0, longest=2048, D=5120, W=4, wide=True),
        # generation: 64 requests through a layer of 5120 channels
        dict(name="step_64", kind="step", dtype="bf16", S=64, D=5120, N=16, wide=True),
        # a large serving batch in binary16
        dict(name="step_512_fp16", kind="step", dtype="fp16", S=512, D=4096, N=16, wide=True),
        # a mixed batch as a server schedules it: a few prompts (some of them continued) and many requests of a few tokens; the
        # batch's buffers are longer than what is in them
        dict(name="scan_mixed_fp16", kind="scan", dtype="fp16", S=48, T=8191, spare=65, longest=2048, D=2048, N=16, wide=True, carried=True),
        # one long prompt through a layer of 5120 channels
        dict(name="scan_long", kind="scan", dtype="bf16", S=1, T=16384, spare=0, longest=16384, D=5120, N=16, wide=True, carried=False),
        # gradients of a small odd layer in binary32
        dict(name="scan_bwd_fp32", kind="scan_bwd", dtype="fp32", S=7, T=517, spare=0, longest=200, D=192, N=16, wide=False),
        # gradients of a packed training batch of documents
        dict(name="scan_bwd_documents", kind="scan_bwd", dtype="bf16", S=11, T=8192, spare=0, longest=2048, D=2048, N=16, wide=True),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["plan", "conv", "conv_bwd", "step", "scan", "scan", "scan_bwd", "scan_bwd"])
    case = dict(kind=kind)
    if kind == "plan":
        S = _spread(rng, 3, 4000)
        longest = _spread(rng, 4, 4096)
        T = rng.randint(max(1, S * longest // 3), max(2, S * longest // 2)) if S * longest < 500000 else rng.randint(50000, 262144)
        case.update(S=S, T=min(T, 262144), spare=rng.choice([0, rng.randint(1, 50)]), longest=longest, tile=2 ** rng.randint(4, 11))
        case["longest"] = max(case["longest"], -(-case["T"] // S))
        return case
    case["dtype"] = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    case["wide"] = rng.random() < 0.5
    D = _spread(rng, 48, 5120)
    case["D"] = D if rng.random() < 0.4 else (D + 63) // 64 * 64
    if kind == "step":
        case.update(S=_spread(rng, 1, 400), N=rng.choice([16, 16, 16, 8, 5, 32, 64]))
        case["S"] = max(1, min(case["S"], int(512 * 4096 * 16 / (case["D"] * case["N"]))))
        return case
    S = _spread(rng, 1, 64)
    longest = _spread(rng, 1, 6000)
    T = max(S, rng.randint((S * longest + 2) // 3, S * longest))
    room = {"conv": MOST / 2, "conv_bwd": MOST / 2, "scan": MOST / 4, "scan_bwd": 8192 * 2048 / 2}[kind]
    if kind in ("scan", "scan_bwd"):
        N = rng.choice([16, 16, 16, 8, 5, 24])
        case["N"] = N
        room = room * 16 / max(N, 16)
    else:
        case["W"] = rng.choice([4, 4, 3, 2])
    T = max(1, min(T, int(room / case["D"])))
    case.update(S=min(S, T), T=T)
    case["longest"] = min(STEPS, max(longest, -(-T // case["S"])))
    case["spare"] = 0 if kind.endswith("bwd") else rng.choice([0, 0, rng.randint(1, 40)])
    if not kind.endswith("bwd"):
        case["carried"] = rng.random() < 0.6
    return case


# ------------------------------------------------------------------------------------------------------- inputs
def _lengths(case, g):
    """S lengths that add up to T, none above `longest`; some are 0 where the batch is large and not full."""
    S, T, longest = case["S"], case["T"], case["longest"]
    if T == S * longest:
        return [longest] * S
    w = (torch.rand(S, generator=g) * 3).exp().tolist()          # a factor of 20 between the shortest and the longest
    if S >= 16:
        for i in range(3, S, 11):
            w[i] = 0.0
    total = sum(w)
    out = [min(longest, int(T * x / total)) for x in w]
    left = T - sum(out)
    order = [i for i in torch.randperm(S, generator=g).tolist() if w[i] > 0.0]
    order += [i for i in range(S) if w[i] == 0.0]                # (only where the others are full)
    for i in order:
        if left == 0:
            break
        more = min(longest - out[i], max(1, left // 2) if i != order[-1] else left)
        out[i] += more
        left -= more
    for i in order:
        more = min(longest - out[i], left)
        out[i] += more
        left -= more
    assert left == 0
    return out


def _rows(g, dev, n, D, dtype, wide, scale=1.0):
    """[n, D] of normal values: by themselves, or as the second half of rows twice as long, as a projection writes them."""
    t = (torch.randn(n, 2 * D if wide else D, generator=g, device=dev) * scale).to(dtype)
    return t[:, D:] if wide else t


def _inputs(case, seed):
    """What the call has to work on, from the seed alone."""
    dev = torch.device("cuda")
    cpu = torch.Generator().manual_seed(seed)
    g = torch.Generator(device=dev).manual_seed(seed)
    kind = case["kind"]
    v = dict(case=case)
    if kind != "step":
        lengths = _lengths(case, cpu)
        v["longest"] = max(lengths)
        v["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=dev)
        v["rows"] = case["T"] + case["spare"]
        if kind == "plan":
            return v
        rows = v["rows"]
    else:
        rows = case["S"]
    dt, D, S = DTYPES[case["dtype"]], case["D"], case["S"]
    if kind in ("conv", "conv_bwd"):
        W = case["W"]
        v["x"] = _rows(g, dev, rows, D, dt, case["wide"])
        bound = 1 / math.sqrt(W)                                  # a depthwise convolution's usual initialisation
        v["weight"] = (torch.rand(D, W, generator=g, device=dev) * 2 - 1) * bound
        v["bias"] = (torch.rand(D, generator=g, device=dev) * 2 - 1) * bound
        if kind == "conv_bwd":
            v["du"] = _rows(g, dev, rows, D, dt, False, 0.1)
            return v
        v["pool"] = torch.randn(2 * S, D, W - 1, generator=g, device=dev).to(dt)
        v["u"] = torch.zeros(rows, D, dtype=dt, device=dev)
    else:
        N = case["N"]
        v["u"] = _rows(g, dev, rows, D, dt, False)
        v["delta"] = _rows(g, dev, rows, D, dt, False, 0.5)
        bc = torch.randn(rows, 2 * N + 7, generator=g, device=dev).to(dt)      # rows of a projection: step rank, B, C
        v["Bm"], v["Cm"] = bc[:, 7:7 + N], bc[:, 7 + N:]
        v["A"] = -torch.exp(torch.randn(D, N, generator=g, device=dev) * 0.5) * torch.arange(1, N + 1, device=dev) / 2
        v["Dv"] = torch.randn(D, generator=g, device=dev)
        v["z"] = _rows(g, dev, rows, D, dt, case["wide"])
        v["bias"] = math.log(1e-3) + torch.rand(D, generator=g, device=dev) * math.log(100.0)     # step sizes of 1e-3 to 1e-1
        if kind == "scan_bwd":
            v["dy"] = _rows(g, dev, rows, D, dt, False, 0.1)
            return v
        v["pool"] = torch.randn(2 * S, D, N, generator=g, device=dev)
        v["y"] = torch.zeros(rows, D, dtype=dt, device=dev)
    # states are read from one half of the pool and left in the other, in no order (a server that keeps a prompt's state to fork it);
    # slot -1: the sequence begins from zero
    slots = torch.randperm(2 * S, generator=cpu).tolist()
    read, write = slots[:S], slots[S:]
    if not case.get("carried", True):
        read = [-1] * S
    elif S > 4:
        read = [-1 if i % 5 == 2 else s for i, s in enumerate(read)]
    v["slots"] = torch.tensor(read, dtype=torch.int32, device=dev)
    v["slots_out"] = torch.tensor(write, dtype=torch.int32, device=dev)
    return v


def prepare(case, seed):
    v = _inputs(case, seed)
    if own:
        import paper_2604_10597_amd as corey
        v["corey"] = corey
        if case["kind"] not in ("plan", "step"):                  # one index serves every layer that the batch goes through
            tile = corey.corey_pack_tile(case["S"], v["rows"], case["D"], case.get("N", 16), backward=case["kind"].endswith("bwd"))
            v["pack"] = corey.corey_pack_plan(v["lengths"], v["rows"], tile)
    return v


# ------------------------------------------------------------------------------------------------------- one pass
def run(state):
    return (_run_own if own else _PLAIN[state["case"]["kind"]])(state)


def _run_own(v):
    corey, kind = v["corey"], v["case"]["kind"]
    if kind == "plan":
        p = corey.corey_pack_plan(v["lengths"], v["rows"], v["case"]["tile"])
        return p.starts, p.seq, p.tiles, p.blocks
    if kind == "conv":
        corey.corey_conv_packed(v["x"], v["weight"], v["bias"], v["pack"], state=v["pool"], slots=v["slots"], slots_out=v["slots_out"], u=v["u"])
        return v["u"], v["pool"]
    if kind == "conv_bwd":
        return corey.corey_conv_packed_bwd(v["x"], v["weight"], v["bias"], v["du"], v["pack"])
    if kind == "scan":
        corey.corey_scan_packed(v["u"], v["delta"], v["A"], v["Bm"], v["Cm"], v["pack"], Dv=v["Dv"], z=v["z"], delta_bias=v["bias"],
                                state=v["pool"], slots=v["slots"], slots_out=v["slots_out"], y=v["y"])
        return v["y"], v["pool"]
    if kind == "step":
        corey.corey_scan_packed_step(v["pool"], v["slots"], v["u"], v["delta"], v["A"], v["Bm"], v["Cm"], Dv=v["Dv"], z=v["z"],
                                     delta_bias=v["bias"], slots_out=v["slots_out"], y=v["y"])
        return v["y"], v["pool"]
    g = corey.corey_scan_packed_bwd(v["u"], v["delta"], v["A"], v["Bm"], v["Cm"], v["pack"], v["dy"], Dv=v["Dv"], z=v["z"],
                                    delta_bias=v["bias"])
    return tuple(g[k] for k in _GRADIENTS)


_GRADIENTS = ("du", "ddelta", "dA", "dB", "dC", "dD", "dz", "ddelta_bias")


# ------------------------------------------------------------------------------------------------------- plain forms
def _pieces(lengths, starts, size, room):
    """The table of pieces of at most `size` tokens: sequence, first token, tokens, bits (1 the sequence's first, 2 its last)."""
    S, dev = lengths.numel(), lengths.device
    n = (lengths + size - 1) // size
    ends = torch.cumsum(n, 0)
    row = torch.arange(room, device=dev)
    s = torch.searchsorted(ends, row, right=True)
    used = s < S
    s = s.clamp(max=S - 1)
    k = row - (ends - n)[s]
    count = torch.minimum(lengths[s] - k * size, torch.full_like(k, size))
    bits = (k == 0).long() + 2 * (k == n[s] - 1).long()
    t = torch.stack([s, starts[s] + k * size, count, bits], 1)
    none = torch.tensor([-1, 0, 0, 0], device=dev)
    return torch.where(used[:, None], t, none).to(torch.int32)


def _starts(lengths):
    return torch.cat([lengths.new_zeros(1, dtype=torch.int64), torch.cumsum(lengths, 0)])


def _plain_plan(v):
    lengths, rows, S, tile = v["lengths"].long(), v["rows"], v["case"]["S"], v["case"]["tile"]
    starts = _starts(lengths)
    t = torch.arange(rows, device=lengths.device)
    seq = torch.searchsorted(starts[1:], t, right=True)
    seq = torch.where(t < starts[S], seq, -1)
    few = min(S, rows)
    return (starts.to(torch.int32), seq.to(torch.int32), _pieces(lengths, starts, tile, rows // tile + few),
            _pieces(lengths, starts, BLOCK, rows // BLOCK + few))


def _padded(v):
    """Index of the padded batch [longest, S]: the row of each token, and whether there is one."""
    lengths = v["lengths"].long()
    starts = _starts(lengths)
    t = torch.arange(v["longest"], device=lengths.device)[:, None]
    return torch.where(t < lengths, starts[:-1] + t, 0), t < lengths, lengths, starts


def _read_slots(pool, slots):
    have = (slots >= 0).view(-1, *[1] * (pool.dim() - 1))
    return torch.where(have, pool[slots.clamp(min=0).long()].float(), torch.zeros((), device=pool.device))


def _taps(v):
    """[T, D, W] inputs of every token's taps in binary32 and, per token, its sequence; inputs before a sequence from its state."""
    lengths, W, T = v["lengths"].long(), v["weight"].shape[1], v["case"]["T"]
    starts = _starts(lengths)
    seq = torch.repeat_interleave(torch.arange(lengths.numel(), device=lengths.device), lengths, output_size=T)
    pos = torch.arange(T, device=lengths.device) - starts[seq]
    x = v["x"][:T].float()
    before = _read_slots(v["pool"], v["slots"]) if "pool" in v else None
    taps = []
    for k in range(W):
        back = W - 1 - k
        tap = torch.zeros_like(x)
        tap[back:] = x[:T - back] if back else x
        early = 0.0 if before is None or not back else before[seq, :, (pos + W - 1 - back).clamp(max=W - 2)]
        taps.append(torch.where((pos >= back)[:, None], tap, early))
    return taps, seq, pos, lengths, starts, before


def _plain_conv(v):
    taps, _, _, lengths, starts, before = _taps(v)
    weight, W, T = v["weight"], v["weight"].shape[1], v["case"]["T"]
    s = v["bias"].expand_as(taps[0])
    for k in range(W):
        s = s + weight[:, k] * taps[k]
    v["u"][:T] = (s * torch.sigmoid(s)).to(v["u"].dtype)
    x = v["x"].float()
    new = []
    for j in range(W - 1):                                        # the last W - 1 inputs; a short sequence keeps some of the old ones
        at = lengths - (W - 1) + j
        old = torch.gather(before, 2, (at + W - 1).clamp(0, W - 2).view(-1, 1, 1).expand(-1, before.shape[1], 1))[:, :, 0]
        new.append(torch.where((at >= 0)[:, None], x[(starts[:-1] + at.clamp(min=0)).clamp(max=T - 1)], old))
    new = torch.stack(new, 2).to(v["pool"].dtype)
    out = v["slots_out"].long()
    v["pool"][out] = torch.where((lengths > 0).view(-1, 1, 1), new, v["pool"][out])
    return v["u"], v["pool"]


def _plain_conv_bwd(v):
    taps, seq, pos, lengths, _, _ = _taps(v)
    weight, W, T = v["weight"], v["weight"].shape[1], v["case"]["T"]
    s = v["bias"].expand_as(taps[0])
    for k in range(W):
        s = s + weight[:, k] * taps[k]
    sig = torch.sigmoid(s)
    dv = v["du"].float() * sig * (1 + s * (1 - sig))
    to_end = (lengths[seq] - 1 - pos)[:, None]
    dx = torch.zeros_like(dv)
    for k in range(W):
        ahead = W - 1 - k
        part = torch.zeros_like(dv)
        part[:T - ahead] = dv[ahead:] if ahead else dv
        dx += weight[:, k] * torch.where(to_end >= ahead, part, 0.0)
    dweight = torch.stack([(dv * taps[k]).double().sum(0) for k in range(W)], 1).float()
    return dx.to(v["x"].dtype), dweight, dv.double().sum(0).float()


def _step_sizes(v, rows):
    return torch.nn.functional.softplus(v["delta"][rows].float() + v["bias"], threshold=60.0)


def _plain_scan(v):
    rows, real, lengths, _ = _padded(v)
    dl = _step_sizes(v, rows) * real[:, :, None]                  # no step where there is no token: the state stays
    u, z = v["u"][rows].float(), v["z"][rows].float()
    Bm, Cm, A = v["Bm"][rows].float(), v["Cm"][rows].float(), v["A"]
    h = _read_slots(v["pool"], v["slots"])
    y = torch.empty_like(u)
    for t in range(rows.shape[0]):
        d = dl[t].unsqueeze(-1)
        h = torch.exp(d * A) * h + (d * u[t].unsqueeze(-1)) * Bm[t].unsqueeze(1)
        y[t] = (h * Cm[t].unsqueeze(1)).sum(-1)
    y = (y + v["Dv"] * u) * (z * torch.sigmoid(z))
    v["y"][:v["case"]["T"]] = torch.zeros_like(v["y"][:v["case"]["T"]]).index_put_((rows[real],), y[real].to(v["y"].dtype))
    out = v["slots_out"].long()
    v["pool"][out] = torch.where((lengths > 0).view(-1, 1, 1), h, v["pool"][out])
    return v["y"], v["pool"]


def _plain_step(v):
    rows = slice(None)
    dl = _step_sizes(v, rows).unsqueeze(-1)
    u, z = v["u"].float(), v["z"].float()
    h = torch.exp(dl * v["A"]) * _read_slots(v["pool"], v["slots"]) + dl * u.unsqueeze(-1) * v["Bm"].float().unsqueeze(1)
    y = (h * v["Cm"].float().unsqueeze(1)).sum(-1) + v["Dv"] * u
    v["y"][:] = (y * (z * torch.sigmoid(z))).to(v["y"].dtype)
    v["pool"][v["slots_out"].long()] = h
    return v["y"], v["pool"]


def _plain_scan_bwd(v):
    rows, real, _, _ = _padded(v)
    real3 = real[:, :, None]
    raw = v["delta"][rows].float() + v["bias"]
    dl = _step_sizes(v, rows) * real3
    u, z, dy = v["u"][rows].float(), v["z"][rows].float(), v["dy"][rows].float() * real3
    Bm, Cm, A = v["Bm"][rows].float(), v["Cm"][rows].float(), v["A"]
    steps, S, D = u.shape
    N = A.shape[1]
    sig = torch.sigmoid(z)
    ds = dy * z * sig
    h = torch.zeros(S, D, N, device=u.device)
    hs = torch.empty(steps, S, D, N, device=u.device)             # the state before every step
    s = torch.empty_like(u)
    for t in range(steps):
        hs[t] = h
        d = dl[t].unsqueeze(-1)
        h = torch.exp(d * A) * h + (d * u[t].unsqueeze(-1)) * Bm[t].unsqueeze(1)
        s[t] = (h * Cm[t].unsqueeze(1)).sum(-1)
    s = s + v["Dv"] * u
    dz = dy * s * sig * (1 + z * (1 - sig))
    g = torch.zeros_like(h)
    ddl, du = torch.empty_like(u), torch.empty_like(u)
    dB, dC = torch.empty_like(Bm), torch.empty_like(Cm)
    dA = torch.zeros(D, N, dtype=torch.float64, device=u.device)
    for t in range(steps - 1, -1, -1):
        d, b = dl[t].unsqueeze(-1), Bm[t].unsqueeze(1)
        kept = torch.exp(d * A) * hs[t]
        dC[t] = (ds[t].unsqueeze(-1) * (kept + d * u[t].unsqueeze(-1) * b)).sum(1)
        g = g + ds[t].unsqueeze(-1) * Cm[t].unsqueeze(1)
        gb = (g * b).sum(-1)
        gk = g * kept
        dB[t] = (g * (d * u[t].unsqueeze(-1))).sum(1)
        du[t] = v["Dv"] * ds[t] + dl[t] * gb
        ddl[t] = gb * u[t] + (gk * A).sum(-1)
        dA += (gk * d).sum(0)
        g = g * torch.exp(d * A)
    draw_ = ddl * torch.sigmoid(raw) * real3
    T = v["case"]["T"]

    def packed(t, like):
        out = torch.empty(T, t.shape[-1], dtype=like.dtype, device=t.device)
        out[rows[real]] = t[real].to(like.dtype)
        return out

    return (packed(du, v["u"]), packed(draw_, v["delta"]), dA.float(), packed(dB, v["Bm"]), packed(dC, v["Cm"]),
            (ds * u).double().sum((0, 1)).float(), packed(dz, v["z"]), draw_.double().sum((0, 1)).float())


_PLAIN = {"plan": _plain_plan, "conv": _plain_conv, "conv_bwd": _plain_conv_bwd, "scan": _plain_scan, "step": _plain_step,
          "scan_bwd": _plain_scan_bwd}


# ------------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    v = _inputs(case, seed)
    return _EXACT[case["kind"]](case, v)


def _exact_plan(case, v):
    lengths, rows, S, tile = v["lengths"].tolist(), v["rows"], case["S"], case["tile"]
    starts, seq, tables = [0], [], ([], [])
    for i, n in enumerate(lengths):
        for table, size in zip(tables, (tile, BLOCK)):
            for k in range(0, n, size):
                table.append([i, starts[-1] + k, min(size, n - k), (k == 0) + 2 * (k + size >= n)])
        seq += [i] * n
        starts.append(starts[-1] + n)
    seq += [-1] * (rows - len(seq))
    for table, size in zip(tables, (tile, BLOCK)):
        table += [[-1, 0, 0, 0]] * (rows // size + min(S, rows) - len(table))
    return tuple(torch.tensor(t, dtype=torch.int32, device=v["lengths"].device) for t in (starts, seq, *tables))


def _sequences(v):
    at = 0
    for i, n in enumerate(v["lengths"].tolist()):
        yield i, slice(at, at + n), n
        at += n


def _silu_and_slope(s):
    sig = 1 / (1 + torch.exp(-s))
    return s * sig, sig + s * sig * (1 - sig)


def _exact_conv(case, v):
    """Sequence by sequence: the inputs with what stood before them, and a window of W of them for every token."""
    W = case["W"]
    w = v["weight"].double()
    backward = "du" in v
    u = v["du"].new_zeros(v["rows"], case["D"]).double() if backward else v["u"].double()
    dw, db = torch.zeros_like(w), torch.zeros_like(w[:, 0])
    pool = None if backward else v["pool"].double()
    slots = None if backward else (v["slots"].tolist(), v["slots_out"].tolist())
    for i, at, n in _sequences(v):
        if n == 0:
            continue
        x = v["x"][at].double().t()                                # [D, n]
        first = torch.zeros_like(w[:, 1:]) if backward or slots[0][i] < 0 else v["pool"][slots[0][i]].double()
        window = torch.cat([first, x], 1).unfold(1, W, 1)          # [D, n, W]
        s, slope = _silu_and_slope((window * w[:, None]).sum(-1) + v["bias"].double()[:, None])
        if backward:
            dv = v["du"][at].double().t() * slope
            dw += (dv[:, :, None] * window).sum(1)
            db += dv.sum(1)
            spread = torch.nn.functional.pad(dv, (0, W - 1)).unfold(1, W, 1)
            u[at] = (spread * w.flip(1)[:, None]).sum(-1).t()
        else:
            u[at] = s.t()
            pool[slots[1][i]] = torch.cat([first, x], 1)[:, n:]
    return (u, dw, db) if backward else (u, pool)


def _joined(a, b, longest):
    """h_t = a_t h_{t-1} + b_t along the first axis by doubling: after k rounds every h holds its last 2^k terms."""
    a, b, step = a.clone(), b.clone(), 1
    while step < longest:
        b[step:] = a[step:] * b[:-step] + b[step:]
        a[step:] = a[step:] * a[:-step]
        step *= 2
    return b


def _exact_scan(case, v):
    """Channel block by channel block over all tokens at once; the decay into a sequence's first token is 0."""
    if case["kind"] == "step":
        v["lengths"] = torch.ones(case["S"], dtype=torch.int32, device=v["u"].device)
    backward = "dy" in v
    T, D, N = sum(v["lengths"].tolist()), case["D"], case["N"]
    dev = v["u"].device
    Bm, Cm, A = v["Bm"][:T].double(), v["Cm"][:T].double(), v["A"].double()
    longest = max(v["lengths"].tolist())
    spans = [(i, at.start, at.stop) for i, at, n in _sequences(v) if n]
    first = torch.tensor([f for _, f, _ in spans], device=dev)
    last = torch.tensor([e - 1 for _, _, e in spans], device=dev)
    ids = [i for i, _, _ in spans]
    if not backward:
        y, pool = v["y"].double(), v["pool"].double()
        read = [v["slots"].tolist()[i] for i in ids]
        into = torch.tensor([v["slots_out"].tolist()[i] for i in ids], device=dev)
    grads = {k: torch.zeros(T, D, dtype=torch.float64, device=dev) for k in ("du", "ddelta", "dz")}
    grads["dB"], grads["dC"] = torch.zeros_like(Bm), torch.zeros_like(Cm)
    grads["dA"], grads["dD"], grads["ddelta_bias"] = torch.zeros_like(A), torch.zeros_like(A[:, 0]), torch.zeros_like(A[:, 0])
    wide = max(1, min(D, int(1.2e8 / (T * N))))
    for c in range(0, D, wide):
        d = slice(c, min(D, c + wide))
        raw = v["delta"][:T, d].double() + v["bias"][d].double()
        dl = torch.clamp(raw, min=0) + torch.log1p(torch.exp(-raw.abs()))
        u = v["u"][:T, d].double()
        gate, slope = _silu_and_slope(v["z"][:T, d].double())
        decay = torch.exp(dl[:, :, None] * A[d])
        b = (dl * u)[:, :, None] * Bm[:, None]
        if not backward:
            h0 = torch.stack([v["pool"][r, d].double() if r >= 0 else torch.zeros_like(A[d]) for r in read])
            b[first] += decay[first] * h0
        cut = decay.clone()
        cut[first] = 0
        h = _joined(cut, b, longest)
        s = (h * Cm[:, None]).sum(-1) + v["Dv"][d].double() * u
        if not backward:
            y[:T, d] = s * gate
            pool[into, d] = h[last]
            continue
        dy = v["dy"][:T, d].double()
        ds = dy * gate
        later = torch.zeros_like(decay)                            # the decay out of a token, into the next of its sequence
        later[:-1] = cut[1:]
        g = _joined(later.flip(0), (ds[:, :, None] * Cm[:, None]).flip(0), longest).flip(0)
        before = torch.zeros_like(h)
        before[1:] = h[:-1]
        through = g * cut * before
        gb = (g * Bm[:, None]).sum(-1)
        draw_ = (gb * u + (through * A[d]).sum(-1)) / (1 + torch.exp(-raw))
        grads["du"][:, d] = v["Dv"][d].double() * ds + dl * gb
        grads["ddelta"][:, d] = draw_
        grads["dz"][:, d] = dy * s * slope
        grads["dA"][d] = (through * dl[:, :, None]).sum(0)
        grads["dB"] += (g * (dl * u)[:, :, None]).sum(1)
        grads["dC"] += (h * ds[:, :, None]).sum(1)
        grads["dD"][d] = (ds * u).sum(0)
        grads["ddelta_bias"][d] = draw_.sum(0)
    return tuple(grads[k] for k in _GRADIENTS) if backward else (y, pool)


_EXACT = {"plan": _exact_plan, "conv": _exact_conv, "conv_bwd": _exact_conv, "scan": _exact_scan, "step": _exact_scan,
          "scan_bwd": _exact_scan}


# ------------------------------------------------------------------------------------------------------- work
def work(case):
    """Each input read once and each output written once; of a recurrence per token, channel and state one exponential (counted
    as one operation), a product for its argument, the update (3) and the read-out (2), backward 10 more."""
    S, kind = case["S"], case["kind"]
    if kind == "plan":
        rows, few = case["T"] + case["spare"], min(S, case["T"] + case["spare"])
        pieces = rows // case["tile"] + rows // BLOCK + 2 * few
        return {"bytes": 4 * S + 4 * (S + 1) + 4 * rows + 16 * pieces, "flops": 0}
    e, D = SIZE[case["dtype"]], case["D"]
    T = case.get("T", S)
    if kind.startswith("conv"):
        W = case["W"]
        if kind == "conv":
            read = 1 if case["carried"] else 0
            return {"bytes": 2 * T * D * e + 4 * D * (W + 1) + (1 + read) * S * D * (W - 1) * e, "flops": T * D * (2 * W + 4)}
        return {"bytes": 3 * T * D * e + 8 * D * (W + 1), "flops": T * D * (6 * W + 9)}
    N = case["N"]
    shared = 4 * D * (N + 2)
    if kind == "scan_bwd":
        return {"bytes": 7 * T * D * e + 4 * T * N * e + 2 * shared, "flops": T * D * (17 * N + 30)}
    states = (2 if case.get("carried", True) else 1) * S * D * N * 4
    return {"bytes": 4 * T * D * e + 2 * T * N * e + shared + states, "flops": T * D * (7 * N + 14)}
