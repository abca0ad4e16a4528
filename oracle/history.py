"""The history block in float64, written from the formulas (numpy): gated recurrence, dropout, rows by expert."""
from __future__ import annotations

import numpy as np

U32 = 2.0 ** -24


def runs(sequence_of, rows, sequences):
    """(sequence, first row, row behind the last) of every run of rows of one sequence."""
    if sequence_of is None:
        n = rows // sequences
        return [(b, b * n, (b + 1) * n) for b in range(sequences)] if n else []
    out, r = [], 0
    s = np.asarray(sequence_of)
    while r < rows:
        e = r + 1
        while e < rows and s[e] == s[r]:
            e += 1
        if 0 <= s[r] < sequences:
            out.append((int(s[r]), r, e))
        r = e
    return out


def sequence_rows(offsets, rows):
    out = np.full(rows, -1, np.int32)
    for b in range(len(offsets) - 1):
        out[max(0, offsets[b]):max(0, min(rows, offsets[b + 1]))] = b
    return out


def sigmoid(x):
    """sigmoid(x), sigmoid(-x)."""
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x)), 1.0 / (1.0 + np.exp(x))


def scan_fwd(gate, value, free, found, initial=None, final=None):
    """h, the state before each row, final (a copy with the runs' last states), and how far a float32 evaluation may be off:

    e = exp(-gate) is 2^t with t = gate log2(e) rounded (1.25 |gate| U32 of e: the product, and the constant's own quarter) and
    exp2's 2 U32; f = 1 / (1 + e) and 1 - f = e f get f (1 - f) of that, and 1 (the sum) + 2 (the reciprocal) + 1 (the product) + 2
    (exp2) U32 of themselves.  A step f h + u adds two roundings: at most 12 U32 of what it sums and, from the first part,
    1.25 |gate| f (1 - f) U32 (|h| + |value|) (|h| alone where u is value).  What was off before shrinks with f like the state
    itself; stretches joined by h -> A h + S add at most 64 roundings of the whole."""
    gate, value = np.asarray(gate, np.float64), np.asarray(value, np.float64)
    h, prev = np.zeros_like(gate), np.zeros_like(gate)
    size, off, prev_size, prev_off = (np.zeros_like(gate) for _ in range(4))
    last = None if final is None else np.array(final, np.float64)
    last_off = None if final is None else np.zeros_like(last)
    f, rest = sigmoid(gate)
    u = value if free else rest * value
    with np.errstate(invalid="ignore"):
        tilt = 1.25 * U32 * np.nan_to_num(np.abs(gate) * f * rest, nan=0.0)        # (inf * 0: open or shut, exactly)
    for b, lo, hi in found:
        x = np.zeros(gate.shape[1]) if initial is None else np.asarray(initial[b], np.float64)
        s, o = np.abs(x), np.zeros_like(x)
        for r in range(lo, hi):
            prev[r], prev_size[r], prev_off[r] = x, s, o
            o = f[r] * o + tilt[r] * (s + (0 if free else np.abs(value[r])))
            x = f[r] * x + u[r]
            s = f[r] * s + np.abs(u[r])
            o = o + 12 * U32 * s
            h[r], size[r], off[r] = x, s, o
        if last is not None:
            last[b], last_off[b] = x, o + 64 * U32 * s
    return dict(h=h, off=off + 64 * U32 * size, prev=prev, prev_size=prev_size, prev_off=prev_off + 64 * U32 * prev_size,
                final=last, final_off=last_off, f=f, rest=rest, tilt=tilt, gate=gate)


def scan_bwd(fwd, value, free, found, dh, dfinal=None, dinitial=None):
    """dgate, dvalue, dinitial and how far each may be off (the same counts; the slope f (1 - f) and the share 1 - f are off by
    at most 1.25 |gate| U32 of themselves besides)."""
    tilt = fwd["tilt"]
    f, rest, value, dh = fwd["f"], fwd["rest"], np.asarray(value, np.float64), np.asarray(dh, np.float64)
    lam, size, off = np.zeros_like(f), np.zeros_like(f), np.zeros_like(f)
    first = None if dinitial is None else np.array(dinitial, np.float64)
    first_off = None if dinitial is None else np.zeros_like(first)
    for b, lo, hi in found:
        m = np.zeros(f.shape[1]) if dfinal is None else np.asarray(dfinal[b], np.float64)
        s, o = np.abs(m), np.zeros_like(m)
        for r in range(hi - 1, lo - 1, -1):
            lam[r], size[r] = dh[r] + m, np.abs(dh[r]) + s
            off[r] = o + 12 * U32 * size[r]
            m, s, o = f[r] * lam[r], f[r] * size[r], f[r] * off[r] + tilt[r] * size[r]
        if first is not None:
            first[b], first_off[b] = m, o + 80 * U32 * s
    off = off + 64 * U32 * size
    there = np.zeros(len(f), bool)
    for _, lo, hi in found:
        there[lo:hi] = True
    with np.errstate(invalid="ignore"):
        slope = f * rest
        d = fwd["prev"] if free else fwd["prev"] - value
        d_size = fwd["prev_size"] + (0 if free else np.abs(value))
        share = np.ones_like(f) if free else rest
        dv, dv_off = lam * share, (off + 12 * U32 * size) * share + (0 if free else tilt * size)
        dg = lam * d * slope
        dg_off = (off * d_size + size * (fwd["prev_off"] + 24 * U32 * d_size)) * slope + tilt * size * d_size
    for a in (dv, dv_off, dg, dg_off):
        a[~there] = 0.0
    return dict(dgate=dg, dgate_off=dg_off, dvalue=dv, dvalue_off=dv_off, dinitial=first, dinitial_off=first_off)


# ------------------------------------------------------------------ dropout

def philox(counter, key):
    """Philox4x32-10 (Salmon et al. 2011): four words from a counter of four and a key of two, uint32 arrays."""
    c = [np.asarray(x, np.uint64) for x in counter]
    k = [int(x) for x in key]
    low, up = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> up) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> up) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def dropout_threshold(p):
    """65536 q."""
    return int(np.floor(float(np.float32(p)) * 65536 + 0.5))


def dropout_keep(rows, cols, p, seed, step, site):
    """[rows][cols]: which elements stay."""
    groups = (cols + 7) // 8
    seed, step = int(seed) % 2 ** 64, int(step) % 2 ** 64
    col = np.broadcast_to(np.arange(groups, dtype=np.uint64) + np.uint64(site << 21), (rows, groups))
    row = np.broadcast_to(np.arange(rows, dtype=np.uint64)[:, None], (rows, groups))
    words = philox([col, row, np.uint64(step % 2 ** 32), np.uint64(step // 2 ** 32)], [seed % 2 ** 32, seed // 2 ** 32])
    half = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=2)
    return half.reshape(rows, groups * 8)[:, :cols] >= np.uint64(dropout_threshold(p))


# ------------------------------------------------------------------ rows by expert

def expert_sort(experts, num_experts, capacity):
    """slot, source, offsets, counts, by one look at each assignment in turn."""
    flat = np.asarray(experts).reshape(-1)
    counts = np.zeros(num_experts, np.int64)
    for e in flat:
        if 0 <= e < num_experts:
            counts[e] += 1
    offsets = np.concatenate([[0], np.cumsum(counts)]) if not capacity else np.arange(num_experts + 1) * capacity
    slot, source = np.full(len(flat), -1), np.full(num_experts * capacity if capacity else len(flat), -1)
    seen = np.zeros(num_experts, np.int64)
    for i, e in enumerate(flat):
        if 0 <= e < num_experts:
            if not capacity or seen[e] < capacity:
                slot[i] = offsets[e] + seen[e]
                source[slot[i]] = i
            seen[e] += 1
    return slot.reshape(np.shape(experts)), source, offsets, counts
