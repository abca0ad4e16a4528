"""The operators of a history block (a layer that mixes a user's history over time and by experts) and what their time is measured on.

A case names one operator and direction ("op"):
  scan_fwd       gated linear recurrence over the rows of each sequence: f = sigmoid(gate), h' = f h + (1 - f) value, or
                 h' = f h + value ("free")
  scan_train     the same keeping what its backward reads, and the gradients of gate, value and initial state
  scan_step      one more row for some of the sequences that a server holds the states of
  dropout_fwd    residual + x with some elements left out, which ones from a counter-based generator
  dropout_bwd    the gradient of x: the same elements left out again
  expert_send    rows ordered by the experts they are sent to, with or without a capacity, and copied there
  expert_back    the experts' rows back at their tokens, weighted and added up
  expert_grad    the gradients: of the experts' rows, of the weights, and of the rows that were sent
and its sizes, types and distributions.  `own` false computes the plain form in elementary torch operations in
float32; `own` true calls the library.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

TORCH_DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ELT = {"f32": 4, "f16": 2, "bf16": 2}
M32 = 0xFFFFFFFF


# ------------------------------------------------------------------------------- the cases


def _scan(op, rows, cols, sequences, layout, dtype, grad=None, carry=False, free=False, pad=0, name=None):
    """layout: "dense" sequences of equal length, "ragged" ones side by side, or "padded" to equal room.
    carry: with initial and final states (and their gradients)."""
    c = dict(op=op, rows=rows, cols=cols, sequences=sequences, layout=layout, dtype=dtype, carry=carry, free=free, pad=pad)
    if op == "scan_train":
        c["grad"] = grad or dtype
    return dict(c, name=name) if name else c


def _step(rows, cols, states, dtype, free=False, name=None):
    c = dict(op="scan_step", rows=rows, cols=cols, states=states, dtype=dtype, free=free)
    return dict(c, name=name) if name else c


def _drop(op, rows, cols, dtype, p, residual=False, pad=0, name=None):
    c = dict(op=op, rows=rows, cols=cols, dtype=dtype, p=p, residual=residual, pad=pad)
    return dict(c, name=name) if name else c


def _expert(op, tokens, cols, k, experts, dtype, factor=0.0, absent=0.0, grad=None, name=None):
    """factor: an expert's room relative to an equal share of the assignments; 0: as much as it is sent."""
    c = dict(op=op, tokens=tokens, cols=cols, k=k, experts=experts, dtype=dtype, factor=factor, absent=absent)
    if op == "expert_grad":
        c["grad"] = grad or dtype
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's history, read when the user arrives: latency
        _scan("scan_fwd", 50, 128, 1, "dense", "bf16", name="scan_one"),
        # the histories of a batch of users, as long as they are, side by side
        _scan("scan_fwd", 131_072, 256, 4_096, "ragged", "bf16", name="scan_ragged"),
        # two event logs of 65536 rows, trained on whole
        _scan("scan_train", 131_072, 512, 2, "dense", "bf16", name="scan_train_long"),
        # a padded batch in float32 with an odd width, states carried from the batch before
        _scan("scan_train", 2_048 * 50, 201, 2_048, "padded", "f32", carry=True, name="scan_train_padded"),
        # the next event of 512 of the 65536 users whose states a server holds
        _step(512, 1_024, 65_536, "f16", name="scan_step"),
        # a training step's activations, added to the path beside them
        _drop("dropout_fwd", 262_144, 256, "bf16", 0.1, residual=True, name="dropout_residual"),
        # a small odd batch
        _drop("dropout_fwd", 77, 1_001, "f32", 0.5, name="dropout_small"),
        # the way back through it, float32 gradients of an odd width
        _drop("dropout_bwd", 65_536, 333, "f32", 0.2, name="dropout_bwd"),
        # the tokens of one request sent to two of eight experts each
        _expert("expert_send", 64, 256, 2, 8, "bf16", name="expert_send_small"),
        # a training batch sent to two of 64 experts each, with a room of 1.25 equal shares
        _expert("expert_send", 65_536, 512, 2, 64, "bf16", factor=1.25, absent=0.05, name="expert_send_room"),
        # four of 32 experts each, and back
        _expert("expert_back", 32_768, 1_024, 4, 32, "bf16", name="expert_back"),
        # its gradients, in float32 as the products' backward leaves them
        _expert("expert_grad", 32_768, 512, 2, 64, "bf16", factor=1.25, grad="f32", name="expert_grad"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cols(rng, lo, hi):
    c = _log(rng, lo, hi)
    return max(lo, c // 16 * 16) if rng.random() < 0.5 else c


def draw(rng: random.Random):
    op = rng.choice(["scan_fwd", "scan_train", "scan_step", "dropout_fwd", "dropout_bwd", "expert_send", "expert_back",
                     "expert_grad"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op in ("scan_fwd", "scan_train"):
        cols = _cols(rng, 16, 2048)
        sequences = _log(rng, 1, 4096)
        most = 2 ** 25 // cols
        length = min(_log(rng, 1, 32_768), max(1, most // sequences))
        return _scan(op, sequences * length, cols, sequences, rng.choice(["dense", "ragged", "padded"]), dtype,
                     grad=rng.choice(["f32", dtype]), carry=rng.random() < 0.5, free=rng.random() < 0.3,
                     pad=rng.choice([0, 0, 8, 5]))
    if op == "scan_step":
        cols, states = _cols(rng, 16, 4096), _log(rng, 1, 65_536)
        states = min(states, 2 ** 26 // cols)
        return _step(min(states, _log(rng, 1, 8192)), cols, states, dtype, free=rng.random() < 0.3)
    if op in ("dropout_fwd", "dropout_bwd"):
        cols = _cols(rng, 16, 8192)
        rows = min(_log(rng, 1, 262_144), 2 ** 26 // cols)
        return _drop(op, rows, cols, dtype, rng.choice([0.05, 0.1, 0.2, 0.5]),
                     residual=op == "dropout_fwd" and rng.random() < 0.5, pad=rng.choice([0, 0, 8, 5]))
    cols, k, experts = _cols(rng, 16, 2048), rng.choice([1, 2, 4, 8]), rng.choice([8, 16, 32, 60, 64, 128, 256])
    tokens = min(_log(rng, 1, 131_072), 2 ** 25 // (cols * k))
    return _expert(op, max(1, tokens), cols, k, experts, dtype, factor=rng.choice([0.0, 0.0, 1.0, 1.25, 2.0]),
                   absent=rng.choice([0.0, 0.1]), grad=rng.choice(["f32", dtype]))


# ------------------------------------------------------------------------------- what a program has in hand


def _randn(g, *shape, dtype, scale=1.0, shift=0.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale + shift).to(dtype)


def _padded(g, rows, cols, pad, dtype, scale=1.0, shift=0.0):
    """[rows][cols] inside rows of cols + pad elements."""
    return _randn(g, rows, cols + pad, dtype=dtype, scale=scale, shift=shift)[:, :cols]


def _lengths(g, case):
    """Rows of each sequence: as geometric lengths are spread, adding up to the case's rows (ragged), or up to an equal room."""
    n, rows = case["sequences"], case["rows"]
    u = -torch.log1p(-torch.rand(n, generator=g, device="cuda", dtype=torch.float64))
    if case["layout"] == "padded":
        room = rows // n
        return torch.clamp((u * room * 0.7).long() + 1, max=room)
    edge = torch.cumsum(u, 0)
    edge = torch.round(edge / edge[-1] * rows).long()
    return torch.diff(edge, prepend=edge.new_zeros(1))


def _sequence_of(g, case):
    """int32 [rows]: each row's sequence, -1 for rows of none; None where all have the same length.  And the longest."""
    n, rows = case["sequences"], case["rows"]
    if case["layout"] == "dense":
        return None, rows // n
    lengths = _lengths(g, case)
    if case["layout"] == "ragged":
        at = torch.repeat_interleave(torch.arange(n, device="cuda"), lengths)
    else:
        b = torch.arange(n, device="cuda")[:, None]
        at = torch.where(torch.arange(rows // n, device="cuda") < lengths[:, None], b, -1).reshape(-1)
    return at.to(torch.int32), int(lengths.max())


def _capacity(case):
    if not case["factor"]:
        return 0
    share = case["tokens"] * case["k"] / case["experts"]
    return max(1, math.ceil(share * case["factor"] / 8) * 8)


def _choices(g, case):
    """int32 [tokens][k]: the experts of each token, some asked for more than others; -1 for tokens that take no part."""
    n, k, E = case["tokens"], case["k"], case["experts"]
    logits = torch.randn(n, E, generator=g, device="cuda") + 0.5 * torch.randn(E, generator=g, device="cuda")
    top = torch.topk(logits, k, dim=1).indices
    if case["absent"]:
        top = torch.where(torch.rand(n, 1, generator=g, device="cuda") < case["absent"], -1, top)
    return top.to(torch.int32).contiguous()


def _ordered(experts, E, capacity):
    """slot [tokens][k], source [rows], offsets [E + 1], counts [E] of the assignments ordered by expert, then as they come."""
    flat = experts.reshape(-1).long()
    m = flat.numel()
    there = flat >= 0
    key = torch.where(there, flat, E)
    order = torch.sort(key, stable=True).indices
    counts = torch.zeros(E + 1, dtype=torch.int64, device="cuda").index_add_(0, key, torch.ones_like(key))[:E]
    begin = torch.cat([counts.new_zeros(1), torch.cumsum(counts, 0)])
    rank = torch.empty_like(flat)
    rank[order] = torch.arange(m, device="cuda") - begin[key[order]]
    if capacity:
        begin = torch.arange(E + 1, device="cuda") * capacity
        there = there & (rank < capacity)
    slot = torch.where(there, begin[key.clamp(max=E - 1)] + rank, -1)
    source = torch.full((E * capacity if capacity else m,), -1, dtype=torch.int64, device="cuda")
    source[slot[there]] = torch.arange(m, device="cuda")[there]
    i32 = torch.int32
    return slot.to(i32).view(experts.shape), source.to(i32), begin.to(i32), counts.to(i32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case=dict(case))
    op, dt = case["op"], TORCH_DTYPE[case["dtype"]]
    f32 = lambda *shape: torch.zeros(*shape, dtype=torch.float32, device="cuda")
    if op in ("scan_fwd", "scan_train"):
        R, C, n = case["rows"], case["cols"], case["sequences"]
        s["sequence_of"], s["longest"] = _sequence_of(g, case)
        s["gate"] = _padded(g, R, C, case["pad"], dt, 2.0, 2.0)           # memories of some ten rows, some far longer
        s["value"] = _padded(g, R, C, case["pad"], dt, 0.3 if case["free"] else 1.0)
        s["h"] = torch.zeros(R, C, dtype=dt, device="cuda")
        s["initial"] = _randn(g, n, C, dtype=torch.float32) if case["carry"] else None
        s["final"] = f32(n, C) if case["carry"] else None
        if op == "scan_train":
            gt = TORCH_DTYPE[case["grad"]]
            s["dh"] = _randn(g, R, C, dtype=gt)
            s["dfinal"] = _randn(g, n, C, dtype=torch.float32) if case["carry"] else None
            s["dgate"], s["dvalue"] = (torch.zeros(R, C, dtype=gt, device="cuda") for _ in range(2))
            s["dinitial"] = f32(n, C) if case["carry"] else None
    elif op == "scan_step":
        R, C, n = case["rows"], case["cols"], case["states"]
        s["gate"], s["value"] = _randn(g, R, C, dtype=dt, scale=2.0, shift=2.0), _randn(g, R, C, dtype=dt)
        s["slots"] = torch.randperm(n, generator=g, device="cuda")[:R].to(torch.int32)
        s["state"] = _randn(g, n, C, dtype=torch.float32)
        s["new_state"], s["h"] = f32(n, C), torch.zeros(R, C, dtype=dt, device="cuda")
    elif op in ("dropout_fwd", "dropout_bwd"):
        R, C = case["rows"], case["cols"]
        s["x"] = _padded(g, R, C, case["pad"], dt)
        s["residual"] = _randn(g, R, C, dtype=dt) if case["residual"] else None
        s["y"] = torch.zeros(R, C, dtype=dt, device="cuda")
        s["rng"] = torch.randint(-2 ** 62, 2 ** 62, (2,), generator=g, device="cuda")     # seed, step
        s["site"] = 3                                                    # which of a model's dropouts
    else:
        n, C, k = case["tokens"], case["cols"], case["k"]
        s["capacity"] = _capacity(case)
        s["experts"] = _choices(g, case)
        s["slot"], s["source"], s["offsets"], s["counts"] = _ordered(s["experts"], case["experts"], s["capacity"])
        rows = s["source"].numel()
        if op == "expert_send":
            s["x"] = _randn(g, n, C, dtype=dt)
            s["out"] = torch.zeros(rows, C, dtype=dt, device="cuda")
            for name in ("slot", "source", "offsets", "counts"):         # what the pass is to find
                s[name] = torch.zeros_like(s[name])
        else:
            s["z"] = _randn(g, rows, C, dtype=dt)
            w = torch.rand(n, k, generator=g, device="cuda") + 0.1
            s["weights"] = w / w.sum(1, keepdim=True)
            if op == "expert_back":
                s["y"] = torch.zeros(n, C, dtype=dt, device="cuda")
            else:
                gt = TORCH_DTYPE[case["grad"]]
                s["dy"], s["drows"] = _randn(g, n, C, dtype=gt), _randn(g, rows, C, dtype=gt)
                s["dz"], s["dweights"] = torch.zeros(rows, C, dtype=gt, device="cuda"), f32(n, k)
                s["dx"] = torch.zeros(n, C, dtype=gt, device="cuda")
    return s


# ------------------------------------------------------------------------------- one pass


def _sigmoids(x):
    """sigmoid(x) and sigmoid(-x)."""
    e = torch.exp(-torch.abs(x))
    r = 1.0 / (1.0 + e)
    return torch.where(x >= 0, r, e * r), torch.where(x >= 0, e * r, r)


def _combined(a, b, longest):
    """b[t] + a[t] (b[t - 1] + a[t - 1] (b[t - 2] + ...)) along the rows, by doubling the distance."""
    d = 1
    while d < longest:
        b = torch.cat([b[:d], b[d:] + a[d:] * b[:-d]])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _ends(s):
    """Per row: its sequence, whether it is there, and whether a sequence starts (ends) with it."""
    c = s["case"]
    at = s["sequence_of"]
    if at is None:
        at = torch.arange(c["sequences"], device="cuda", dtype=torch.int32)
        at = at[:, None].expand(-1, c["rows"] // c["sequences"]).reshape(-1)
    at = at.long()
    there = at >= 0
    change = at[1:] != at[:-1]
    one = torch.ones(1, dtype=torch.bool, device="cuda")
    return at, there, there & torch.cat([one, change]), there & torch.cat([change, one])


def _plain_scan(s):
    c = s["case"]
    dt = s["h"].dtype
    at, there, first, last = _ends(s)
    f, rest = _sigmoids(s["gate"].float())
    v = s["value"].float()
    b = v if c["free"] else rest * v
    b = torch.where(there[:, None], b, 0.0)
    before = None if s["initial"] is None else s["initial"][at[first]]
    if before is not None:
        b[first] = b[first] + f[first] * before
    a = torch.where((there & ~first)[:, None], f, 0.0)
    h = _combined(a, b, s["longest"])
    del a, b
    out = [h.to(dt)]
    if c["carry"]:
        out.append(s["final"].index_copy(0, at[last], h[last]))
    if c["op"] == "scan_fwd":
        return out
    prev = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
    prev[first] = 0.0 if before is None else before
    del h
    dh = torch.where(there[:, None], s["dh"].float(), 0.0)
    if c["carry"]:
        dh[last] = dh[last] + s["dfinal"][at[last]]
    a = torch.cat([f[1:], torch.zeros_like(f[:1])])
    a = torch.where((there & ~last)[:, None], a, 0.0)
    lam = _combined(a.flip(0), dh.flip(0), s["longest"]).flip(0)
    del a, dh
    gt = s["dh"].dtype
    dv = lam if c["free"] else lam * rest
    dg = lam * (prev if c["free"] else prev - v) * f * rest
    zero = there[:, None]
    out += [torch.where(zero, dg, 0.0).to(gt), torch.where(zero, dv, 0.0).to(gt)]
    if c["carry"]:
        out.append(s["dinitial"].index_copy(0, at[first], f[first] * lam[first]))
    return out


def _philox(c0, c1, c2, c3, seed):
    """Philox4x32-10 of 32-bit words held in int64."""
    k0, k1 = seed & M32, (seed >> 32) & M32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & M32) ^ c1 ^ k0, p1 & M32, ((p0 >> 32) & M32) ^ c3 ^ k1, p0 & M32
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    return c0, c1, c2, c3


def _plain_dropout(s):
    c = s["case"]
    R, C = c["rows"], c["cols"]
    groups = (C + 7) // 8
    col = torch.arange(groups, device="cuda") + (s["site"] << 21)
    row = torch.arange(R, device="cuda")[:, None]
    seed, step = s["rng"][0], s["rng"][1]
    words = _philox(col.expand(R, groups), row.expand(R, groups), step & M32, (step >> 32) & M32, seed)
    bits = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], dim=2).view(R, groups * 8)[:, :C]
    most = int(math.floor(c["p"] * 65536 + 0.5))
    y = torch.where(bits >= most, s["x"].float() * (65536.0 / (65536 - most)), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _taken(rows, slot):
    """rows[slot] in float32, zeros where there is no slot."""
    return torch.where((slot >= 0)[:, None], rows[slot.clamp(min=0).long()].float(), 0.0)


def _plain_expert(s):
    c = s["case"]
    k = c["k"]
    if c["op"] == "expert_send":
        slot, source, offsets, counts = _ordered(s["experts"], c["experts"], s["capacity"])
        x = s["x"][torch.div(source.clamp(min=0).long(), k, rounding_mode="floor")]
        return [slot, source, offsets, counts, torch.where((source >= 0)[:, None], x, 0.0)]
    slot, w, z = s["slot"], s["weights"], s["z"]
    if c["op"] == "expert_back":
        y = _taken(z, slot[:, 0]) * w[:, :1]
        for j in range(1, k):
            y = y + _taken(z, slot[:, j]) * w[:, j:j + 1]
        return y.to(z.dtype)
    dy = s["dy"].float()
    dw = torch.stack([(_taken(z, slot[:, j]) * dy).sum(1) for j in range(k)], dim=1)
    at = s["source"].clamp(min=0).long()
    dz = dy[torch.div(at, k, rounding_mode="floor")] * w.reshape(-1)[at][:, None]
    dz = torch.where((s["source"] >= 0)[:, None], dz, 0.0)
    dx = _taken(s["drows"], slot[:, 0])
    for j in range(1, k):
        dx = dx + _taken(s["drows"], slot[:, j])
    return [dz.to(s["dy"].dtype), dw, dx.to(s["dy"].dtype)]


def _plain(s):
    c = s["case"]
    op = c["op"]
    if op in ("scan_fwd", "scan_train"):
        return _plain_scan(s)
    if op == "scan_step":
        at = s["slots"].long()
        f, rest = _sigmoids(s["gate"].float())
        v = s["value"].float()
        h = f * s["state"][at] + (v if c["free"] else rest * v)
        s["new_state"][at] = h
        return [h.to(s["h"].dtype), s["new_state"]]
    if op in ("dropout_fwd", "dropout_bwd"):
        return _plain_dropout(s)
    return _plain_expert(s)


def _scratch(s, name, nbytes):
    """Memory that a program keeps beside its tensors."""
    if name not in s:
        s[name] = torch.empty(max(256, nbytes()), dtype=torch.uint8, device="cuda")
    return s[name]


def _library(s):
    import paper_2403_00877_amd as dmt
    c = s["case"]
    op = c["op"]
    if op in ("scan_fwd", "scan_train"):
        form = "free" if c["free"] else "coupled"
        ws = _scratch(s, "ws", lambda: dmt.dmt_gated_scan_workspace_bytes(c["rows"], c["cols"]))
        where = dict(form=form, sequence_of=s["sequence_of"], sequences=c["sequences"], initial=s["initial"])
        kept = None
        if op == "scan_train":
            kept = _scratch(s, "kept", lambda: dmt.dmt_gated_scan_kept_bytes(c["rows"], c["cols"]))
        dmt.dmt_gated_scan_fwd(s["gate"], s["value"], s["h"], ws, final=s["final"], kept=kept, **where)
        out = [s["h"]] + ([s["final"]] if c["carry"] else [])
        if op == "scan_fwd":
            return out
        dmt.dmt_gated_scan_bwd(s["gate"], s["value"], s["dh"], s["dgate"], s["dvalue"], kept, ws, dfinal=s["dfinal"],
                               dinitial=s["dinitial"], **where)
        return out + [s["dgate"], s["dvalue"]] + ([s["dinitial"]] if c["carry"] else [])
    if op == "scan_step":
        dmt.dmt_gated_scan_step(s["gate"], s["value"], s["state"], s["new_state"], s["h"], slots=s["slots"],
                                form="free" if c["free"] else "coupled")
        return [s["h"], s["new_state"]]
    if op == "dropout_fwd":
        dmt.dmt_dropout_fwd(s["x"], c["p"], s["rng"], s["y"], residual=s["residual"], site=s["site"])
        return s["y"]
    if op == "dropout_bwd":
        dmt.dmt_dropout_bwd(s["x"], c["p"], s["rng"], s["y"], site=s["site"])
        return s["y"]
    if op == "expert_send":
        ws = _scratch(s, "ws", lambda: dmt.dmt_expert_sort_workspace_bytes(c["tokens"], c["k"], c["experts"]))
        dmt.dmt_expert_sort(s["experts"], c["experts"], s["slot"], s["source"], s["offsets"], s["counts"], ws,
                            capacity=s["capacity"])
        dmt.dmt_expert_gather(s["x"], s["slot"], s["source"], s["out"])
        return [s["slot"], s["source"], s["offsets"], s["counts"], s["out"]]
    if op == "expert_back":
        dmt.dmt_expert_combine(s["z"], s["slot"], s["weights"], s["y"])
        return s["y"]
    dmt.dmt_expert_combine_bwd(s["dy"], s["z"], s["slot"], s["source"], s["weights"], s["dz"], s["dweights"])
    dmt.dmt_expert_combine(s["drows"], s["slot"], None, s["dx"])
    return [s["dz"], s["dweights"], s["dx"]]


def run(state):
    return _library(state) if own else _plain(state)


# ------------------------------------------------------------------------------- the definition in 64 bits


def _exact_scan(s):
    """Row after row: at time t the t-th row of every sequence that is that long."""
    c = s["case"]
    at = s["sequence_of"]
    n, R, C = c["sequences"], c["rows"], c["cols"]
    if at is None:
        at = torch.arange(R, device="cuda") // (R // n)
    at = at.long().cpu().numpy()
    begin, length = np.zeros(n, np.int64), np.zeros(n, np.int64)
    rows = np.nonzero(at >= 0)[0]
    np.add.at(length, at[rows], 1)
    begin[at[rows][::-1]] = rows[::-1]                    # the first row of each
    order = np.argsort(-length, kind="stable")
    active = np.searchsorted(-length[order], -np.arange(length.max()), side="left")
    seq = torch.from_numpy(order).cuda()
    start = torch.from_numpy(begin[order]).cuda()
    full = torch.from_numpy(length[order]).cuda()
    f = 1.0 / (1.0 + torch.exp(-s["gate"].double()))
    rest = 1.0 / (1.0 + torch.exp(s["gate"].double()))
    v = s["value"].double()
    u = v if c["free"] else rest * v
    h = torch.zeros(R, C, dtype=torch.float64, device="cuda")
    prev = torch.zeros_like(h)
    zero = torch.zeros(n, C, dtype=torch.float64, device="cuda")
    x = zero if s["initial"] is None else s["initial"].double()[seq]
    for t, m in enumerate(active.tolist()):
        at_t = start[:m] + t
        x = x[:m]
        prev[at_t] = x
        x = f[at_t] * x + u[at_t]
        h[at_t] = x
    some = full > 0
    out = [h]
    if c["carry"]:
        end = s["final"].double().clone()
        end[seq[some]] = h[(start + full - 1)[some]]
        out.append(end)
    if c["op"] == "scan_fwd":
        return out
    dh = s["dh"].double()
    lam = torch.zeros_like(h)
    mu = zero.clone()                                     # f lambda of the row behind, or the final state's gradient
    if c["carry"]:
        mu += s["dfinal"].double()[seq]
    for t in range(len(active) - 1, -1, -1):
        m = int(active[t])
        at_t = start[:m] + t
        x = dh[at_t] + mu[:m]
        lam[at_t] = x
        mu[:m] = f[at_t] * x
    dg = lam * (prev if c["free"] else prev - v) * f * rest
    dv = lam if c["free"] else lam * rest
    out += [dg, dv]
    if c["carry"]:
        first = s["dinitial"].double().clone()
        first[seq[some]] = mu[some]
        out.append(first)
    return out


def _exact_dropout(s):
    """The generator by products of 16-bit halves, on columns of words."""
    c = s["case"]
    R, C = c["rows"], c["cols"]

    def product(m, x):
        ml, mh, xl, xh = m & 0xFFFF, m >> 16, x & 0xFFFF, x >> 16
        mid = ml * xh + (ml * xl >> 16)
        mid2 = mh * xl + (mid & 0xFFFF)
        return mh * xh + (mid >> 16) + (mid2 >> 16), (mid2 & 0xFFFF) << 16 | (ml * xl & 0xFFFF)

    seed, step = (int(v) % 2 ** 64 for v in s["rng"])
    keep = torch.empty(R, C, dtype=torch.bool, device="cuda")
    least = round(c["p"] * 65536)
    row = torch.arange(R, device="cuda")
    for j in range(0, C, 8):
        x = [torch.full_like(row, s["site"] * 2 ** 21 + j // 8), row, torch.full_like(row, step % 2 ** 32),
             torch.full_like(row, step // 2 ** 32)]
        for i in range(10):
            ka, kb = (seed % 2 ** 32 + i * 0x9E3779B9) % 2 ** 32, (seed // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32
            (ha, la), (hb, lb) = product(0xD2511F53, x[0]), product(0xCD9E8D57, x[2])
            x = [hb ^ x[1] ^ ka, lb, ha ^ x[3] ^ kb, la]
        for q in range(min(8, C - j)):
            keep[:, j + q] = (x[q // 2] >> q % 2 * 16) % 65536 >= least
    y = s["x"].double() * keep / (1.0 - least / 65536.0)
    return y if s["residual"] is None else y + s["residual"].double()


def _exact_expert(s):
    c = s["case"]
    k, E, cap = c["k"], c["experts"], s["capacity"]
    experts = s["experts"].cpu().numpy()
    lists = [np.nonzero(experts.reshape(-1) == e)[0] for e in range(E)]
    begin = np.concatenate([[0], np.cumsum([len(v) for v in lists])]) if not cap else np.arange(E + 1) * cap
    slot, source = np.full(experts.size, -1), np.full(s["source"].numel(), -1)
    for e, v in enumerate(lists):
        kept = v[:cap] if cap else v
        slot[kept] = begin[e] + np.arange(len(kept))
        source[begin[e]:begin[e] + len(kept)] = kept
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    full = np.nonzero(source >= 0)[0]
    rows, tokens, pairs = cuda(full), cuda(source[full] // k), cuda(source[full])
    n, C = c["tokens"], c["cols"]
    if c["op"] == "expert_send":
        out = torch.zeros(len(source), C, dtype=torch.float64, device="cuda")
        out[rows] = s["x"].double()[tokens]
        return [cuda(slot.reshape(experts.shape)), cuda(source), cuda(begin), cuda(np.array([len(v) for v in lists])), out]
    w = s["weights"].double().reshape(-1)[pairs]
    z = s["z"].double()[rows]
    if c["op"] == "expert_back":
        return torch.zeros(n, C, dtype=torch.float64, device="cuda").index_add_(0, tokens, z * w[:, None])
    dy = s["dy"].double()[tokens]
    dz = torch.zeros(len(source), C, dtype=torch.float64, device="cuda")
    dz[rows] = dy * w[:, None]
    dw = torch.zeros(n * k, dtype=torch.float64, device="cuda")
    dw[pairs] = (dy * z).sum(1)
    dx = torch.zeros(n, C, dtype=torch.float64, device="cuda").index_add_(0, tokens, s["drows"].double()[rows])
    return [dz, dw.view(n, k), dx]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("scan_fwd", "scan_train"):
        return _exact_scan(s)
    if op == "scan_step":
        at = s["slots"].long()
        g, v = s["gate"].double(), s["value"].double()
        f, rest = 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))
        h = f * s["state"].double()[at] + v * (1.0 if case["free"] else rest)
        new = s["new_state"].double()
        new[at] = h
        return [h, new]
    if op in ("dropout_fwd", "dropout_bwd"):
        return _exact_dropout(s)
    return _exact_expert(s)


# ------------------------------------------------------------------------------- what a pass cannot do without


def work(case):
    op, e = case["op"], ELT[case["dtype"]]
    if op in ("scan_fwd", "scan_train"):
        n = case["rows"] * case["cols"]
        share = 0.5 if case["layout"] == "padded" else 1.0      # of the inputs; outputs are written whole
        state = 4 * case["sequences"] * case["cols"] if case["carry"] else 0
        b = n * e * (2 * share + 1) + 2 * state + (0 if case["layout"] == "dense" else 4 * case["rows"])
        if op == "scan_fwd":
            return {"bytes": b, "flops": 9 * n * share}
        eg = ELT[case["grad"]]
        return {"bytes": b + n * (share * (2 * e + eg) + 2 * eg) + 2 * state, "flops": 30 * n * share}
    if op == "scan_step":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (3 * e + 8) + 4 * case["rows"], "flops": 9 * n}
    if op in ("dropout_fwd", "dropout_bwd"):
        n = case["rows"] * case["cols"]
        return {"bytes": n * e * (3 if case["residual"] else 2) + 16, "flops": 3 * n}
    n, C, k = case["tokens"], case["cols"], case["k"]
    cap = _capacity(case)
    rows = case["experts"] * cap if cap else n * k
    sent = n * k * (1 - case["absent"])
    if cap:
        sent = min(sent, rows)
    if op == "expert_send":
        return {"bytes": n * C * e + rows * C * e + 8 * n * k + 4 * rows, "flops": n * k}
    if op == "expert_back":
        return {"bytes": sent * C * e + n * C * e + 8 * n * k, "flops": 2 * sent * C}
    eg = ELT[case["grad"]]
    return {"bytes": n * C * eg + sent * C * e + rows * C * eg + sent * C * eg + n * C * eg + 12 * n * k + 4 * rows,
            "flops": 4 * sent * C}
