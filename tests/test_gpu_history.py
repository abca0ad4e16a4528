"""The history block's kernels against float64, through the binding.

Tolerances come from the number format and the depth of the sums, before any run: one rounding is off by at most U of its type
(2^-8 bf16, 2^-11 f16, 2^-24 f32) relative to the value; oracle/history.py counts the roundings of the recurrences.
"""
import numpy as np
import pytest
import torch

from oracle import history as hs
from test_gpu_sequence import DT, TINY, U, U32, blank, bytes_buf, close, f64, matrix, untouched

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dmt():
    import paper_2403_00877_amd as d
    return d


def no_bad():
    return torch.full((1,), -1, dtype=torch.int64, device="cuda")


# ------------------------------------------------------------------ gated recurrence

def lengths_of(rng, rows, sequences):
    edge = np.sort(rng.integers(0, rows + 1, sequences - 1)) if sequences > 1 else np.zeros(0, np.int64)
    return np.diff(np.concatenate([[0], edge, [rows]]))


def sequences_of(rng, kind, rows, sequences):
    """int32 [rows] or None."""
    if kind == "equal":
        return None
    order = rng.permutation(sequences)
    if kind == "room":
        room = rows // sequences
        there = np.arange(room) < rng.integers(0, room + 1, sequences)[:, None]
        return np.where(there, order[:, None], -1).reshape(-1).astype(np.int32)
    seq = np.repeat(order, lengths_of(rng, rows, sequences))
    if kind == "holes":                       # rows of no sequence: some stretches, the front, the end; ids past the last
        for _ in range(max(1, rows // 40)):
            at = rng.integers(0, rows)
            seq[at:at + rng.integers(1, 5)] = -1 - rng.integers(0, 2)
        at = rng.integers(0, rows)
        seq[at:at + 2] = sequences + rng.integers(0, 3)
        seq[:min(2, rows // 3)] = -1
        if rows > 3:
            seq[-1] = -7
        # an id's rows lie together: what comes behind a gap is an id of its own or of none
        seen, last = set(), None
        for r in range(rows):
            if seq[r] != last and 0 <= seq[r] < sequences:
                if seq[r] in seen:
                    seq[r] = last if last is not None and not 0 <= last < sequences else -1
                else:
                    seen.add(int(seq[r]))
            last = int(seq[r])
    return seq.astype(np.int32)


#        rows, cols, sequences, pad, shift
SHAPES = [(1, 1, 1, 0, 0), (2, 3, 2, 1, 1), (50, 128, 1, 0, 0), (96, 16, 3, 0, 0), (130, 33, 2, 3, 1), (333, 7, 9, 2, 1),
          (515, 130, 5, 0, 0), (1100, 20, 4, 5, 2), (3000, 65, 3, 0, 0), (2600, 1, 1, 0, 0), (2048, 300, 64, 8, 0),
          (9000, 40, 9, 0, 0)]


def scan_case(dmt, rows, cols, sequences, pad, shift, dtype, gd, kind, free, carry, seed=0):
    rng = np.random.default_rng(rows + 7 * cols + seed)
    seq = sequences_of(rng, kind, rows, sequences)
    if kind == "equal" and rows % sequences:
        rows -= rows % sequences
    gate = matrix(rng, rows, cols, dtype, pad, shift, 3.0, 1.0)
    value = matrix(rng, rows, cols, dtype, pad, shift)
    dh = matrix(rng, rows, cols, gd, pad, shift)
    if rows > 8:                               # gates that are shut or open
        gate[1], gate[rows // 2], gate[5] = -200.0, 200.0, 0.0
        gate[2, 0], gate[rows // 2 + 1, 0] = float("inf"), float("-inf")
    found = hs.runs(seq, rows, sequences)
    there = np.zeros(rows, bool)
    for _, lo, hi in found:
        there[lo:hi] = True
    d_there = torch.from_numpy(~there).cuda()
    for t in (gate, value, dh):
        t[d_there] = float("nan")
    d_seq = None if seq is None else torch.from_numpy(seq).cuda()
    state = lambda: torch.from_numpy(rng.normal(size=(sequences, cols)).astype(np.float32)).cuda()
    initial, dfinal = (state(), state()) if carry else (None, None)
    final, dinitial = (torch.full((sequences, cols), 7.0, device="cuda") for _ in range(2)) if carry else (None, None)
    h, around = blank(rows, cols, dtype, pad, shift)
    kept = torch.full((max(1, dmt.dmt_gated_scan_kept_bytes(rows, cols)),), 0xFF, dtype=torch.uint8, device="cuda")
    ws = bytes_buf(dmt.dmt_gated_scan_workspace_bytes(rows, cols))
    ws.fill_(0xFF)
    bad = no_bad()
    form = "free" if free else "coupled"
    where = dict(form=form, sequence_of=d_seq, sequences=sequences, initial=initial)
    dmt.dmt_gated_scan_fwd(gate, value, h, ws, final=final, kept=kept, first_bad=bad, **where)
    g64, v64 = f64(gate), f64(value)
    ref = hs.scan_fwd(g64, v64, free, found, None if initial is None else f64(initial),
                      None if final is None else np.full((sequences, cols), 7.0))
    close(h, ref["h"], U[dtype] * (np.abs(ref["h"]) + ref["off"]) + ref["off"] + TINY[dtype], "h")
    untouched(around)
    if carry:
        close(final, ref["final"], ref["final_off"] + 1e-37, "final")
    over = np.nonzero(seq >= sequences)[0] if seq is not None else []
    assert int(bad.cpu()) == (over[0] if len(over) else -1)
    h2, _ = blank(rows, cols, dtype, pad, shift)
    ws.fill_(0xA5)
    dmt.dmt_gated_scan_fwd(gate, value, h2, ws, **where)                       # keeping nothing: the same bits
    assert torch.equal(h.contiguous().view(torch.uint8), h2.contiguous().view(torch.uint8))

    dgate, around_g = blank(rows, cols, gd, pad, shift)
    dvalue, around_v = blank(rows, cols, gd, pad + 1, shift)
    ws.fill_(0xFF)
    dmt.dmt_gated_scan_bwd(gate, value, dh, dgate, dvalue, kept, ws, dfinal=dfinal, dinitial=dinitial, **where)
    back = hs.scan_bwd(ref, v64, free, found, f64(dh), None if dfinal is None else f64(dfinal),
                       None if dinitial is None else np.full((sequences, cols), 7.0))
    for name, got in (("dgate", dgate), ("dvalue", dvalue)):
        off = back[name + "_off"]
        close(got, back[name], U[gd] * (np.abs(back[name]) + off) + off + TINY[gd], name)
    untouched(around_g)
    untouched(around_v)
    if carry:
        close(dinitial, back["dinitial"], back["dinitial_off"] + 1e-37, "dinitial")


@pytest.mark.parametrize("dtype,gd", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f32")])
@pytest.mark.parametrize("kind", ["equal", "ragged", "holes"])
@pytest.mark.parametrize("rows,cols,sequences,pad,shift", SHAPES)
def test_gated_scan(dmt, rows, cols, sequences, pad, shift, kind, dtype, gd):
    for free, carry in ((False, True), (True, False)):
        scan_case(dmt, rows, cols, sequences, pad, shift, dtype, gd, kind, free, carry)


@pytest.mark.parametrize("rows,cols,sequences,dtype", [(70_000, 130, 10_000, "bf16"), (66_000, 128, 66_000, "f16"),
                                                       (105_000, 64, 2_100, "f32"), (68_000, 300, 4_000, "f32"),
                                                       (21_840, 1_100, 312, "f32"), (27_300, 3_600, 300, "bf16")])
def test_gated_scan_of_many_equal_sequences(dmt, rows, cols, sequences, dtype):
    scan_case(dmt, rows, cols, sequences, 0, 0, dtype, dtype, "equal", False, True)


@pytest.mark.parametrize("kind", ["room", "ragged"])
@pytest.mark.parametrize("room", [32, 33, 37, 50, 63, 64])
@pytest.mark.parametrize("cols,sequences,dtype", [(300, 60, "bf16"), (70, 90, "f32"), (9, 150, "f16")])
def test_gated_scan_of_padded_rooms(dmt, room, cols, sequences, dtype, kind):
    """Rows in as many equal rooms as sequences, and sequences of any length whose mean is a room."""
    scan_case(dmt, room * sequences, cols, sequences, 0, 0, dtype, dtype, kind, False, True, seed=room)


@pytest.mark.parametrize("kind", ["room", "ragged"])
@pytest.mark.parametrize("room,cols,sequences,dtype", [(33, 230, 1100, "f32"), (50, 520, 400, "bf16"), (61, 129, 1050, "f32")])
def test_gated_scan_of_many_padded_rooms(dmt, room, cols, sequences, dtype, kind):
    """So many that stretches are as long as the rooms; the workspace is of just the size asked for."""
    scan_case(dmt, room * sequences, cols, sequences, 0, 0, dtype, dtype, kind, False, True, seed=room)


@pytest.mark.parametrize("rows,cols,starts", [(400_000, 64, [0]), (400_000, 64, [0, 131, 399_990]), (300_000, 5, [0, 250_000]),
                                              (1_100_000, 20, [0, 1_000_003])])
def test_gated_scan_of_long_sequences(dmt, rows, cols, starts):
    """Open gates and whole numbers: sums of up to 2^20 ones are exact, whatever the rows are cut into."""
    rng = np.random.default_rng(rows)
    seq = np.zeros(rows, np.int32)
    for s in starts[1:]:
        seq[s:] += 1
    gate = torch.full((rows, cols), 100.0, device="cuda")                     # f is 1 to the last bit
    ones = torch.from_numpy(rng.integers(0, 3, (rows, cols)).astype(np.float32)).cuda()
    d_seq = torch.from_numpy(seq).cuda()
    n = len(starts)
    h, final = torch.full((rows, cols), 7.0, device="cuda"), torch.full((n, cols), 7.0, device="cuda")
    kept = bytes_buf(dmt.dmt_gated_scan_kept_bytes(rows, cols))
    ws = bytes_buf(dmt.dmt_gated_scan_workspace_bytes(rows, cols))
    initial = torch.full((n, cols), 5.0, device="cuda")
    where = dict(form="free", sequence_of=d_seq if n > 1 else None, sequences=n, initial=initial)
    dmt.dmt_gated_scan_fwd(gate, ones, h, ws, final=final, kept=kept, **where)
    ends = starts[1:] + [rows]
    for b, (lo, hi) in enumerate(zip(starts, ends)):
        total = torch.cumsum(ones[lo:hi].double(), 0) + 5
        assert torch.equal(h[lo:hi].double(), total) and torch.equal(final[b].double(), total[-1])
    dg, dv = torch.empty_like(h), torch.empty_like(h)
    dinitial, dfinal = torch.full((n, cols), 7.0, device="cuda"), torch.full((n, cols), 3.0, device="cuda")
    dmt.dmt_gated_scan_bwd(gate, ones, ones, dg, dv, kept, ws, dfinal=dfinal, dinitial=dinitial, **where)
    for b, (lo, hi) in enumerate(zip(starts, ends)):
        total = torch.cumsum(ones[lo:hi].double().flip(0), 0).flip(0) + 3
        assert torch.equal(dv[lo:hi].double(), total) and torch.equal(dinitial[b].double(), total[0])


def test_gated_scan_keeps_nan_where_it_is(dmt):
    rows, cols = 2000, 40
    rng = np.random.default_rng(3)
    seq = np.repeat(np.arange(20), 100).astype(np.int32)
    gate, value = matrix(rng, rows, cols, "f32"), matrix(rng, rows, cols, "f32")
    d_seq = torch.from_numpy(seq).cuda()
    outs = []
    for poison in (False, True):
        if poison:
            gate[350, 3], value[360, 4], value[1200, 39], gate[1999, 0] = float("nan"), float("inf"), float("nan"), float("nan")
        h, dg, dv = (torch.empty(rows, cols, device="cuda") for _ in range(3))
        kept, ws = bytes_buf(dmt.dmt_gated_scan_kept_bytes(rows, cols)), bytes_buf(dmt.dmt_gated_scan_workspace_bytes(rows, cols))
        dmt.dmt_gated_scan_fwd(gate, value, h, ws, sequence_of=d_seq, sequences=20, kept=kept)
        dmt.dmt_gated_scan_bwd(gate, value, value.nan_to_num(posinf=1.0), dg, dv, kept, ws, sequence_of=d_seq, sequences=20)
        outs.append((h, dg, dv))
    clean = torch.ones(rows, cols, dtype=torch.bool, device="cuda")
    for s, c in ((3, 3), (3, 4), (12, 39), (19, 0)):
        clean[s * 100:s * 100 + 100, c] = False
    for a, b in zip(*outs):
        assert torch.equal(a[clean], b[clean]) and bool(torch.isfinite(b[clean]).all())
    h = outs[1][0]
    assert bool(torch.isnan(h[350:400, 3]).all()) and bool(torch.isfinite(h[300:350, 3]).all())
    assert bool(torch.isinf(h[360:365, 4]).all()) and bool(torch.isnan(h[1200:1300, 39]).all())


def test_gated_scan_repeats_bit_for_bit(dmt):
    rows, cols = 20_000, 96
    rng = np.random.default_rng(4)
    gate, value = matrix(rng, rows, cols, "bf16", scale=2.0, mean=2.0), matrix(rng, rows, cols, "bf16")
    outs = []
    for _ in range(3):
        h, dg, dv = (torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda") for _ in range(3))
        kept, ws = bytes_buf(dmt.dmt_gated_scan_kept_bytes(rows, cols)), bytes_buf(dmt.dmt_gated_scan_workspace_bytes(rows, cols))
        dmt.dmt_gated_scan_fwd(gate, value, h, ws, kept=kept)
        dmt.dmt_gated_scan_bwd(gate, value, value, dg, dv, kept, ws)
        outs.append([t.view(torch.int16) for t in (h, dg, dv)])
    assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(outs[0], o))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,states,pad,shift", [(1, 1, 1, 0, 0), (3, 5, 9, 1, 1), (70, 1030, 100, 3, 1), (512, 64, 4000, 0, 0),
                                                        (1500, 33, 1500, 0, 0)])
def test_gated_scan_step(dmt, rows, cols, states, pad, shift, dtype):
    rng = np.random.default_rng(rows + cols)
    for kind in ("slots", "holes", "none"):
        if kind == "none" and states < rows:
            continue
        gate, value = matrix(rng, rows, cols, dtype, pad, shift, 3.0), matrix(rng, rows, cols, dtype, pad, shift)
        state = torch.from_numpy(rng.normal(size=(states, cols)).astype(np.float32)).cuda()
        slots = rng.permutation(states)[:rows].astype(np.int32)
        refused = []
        if kind == "holes" and rows > 2:
            slots[rng.random(rows) < 0.2] = -1
            slots[1] = states + 3
            slots[rows // 2] = slots[0] = states - 1                          # named twice: the earlier row has it
            where = np.nonzero(slots == states - 1)[0]
            refused = sorted([1, *where[1:]])
        if kind == "none":
            slots = np.arange(rows, dtype=np.int32)
        for free in (False, True):
            start = f64(state)
            kept = state.clone()
            h, around = blank(rows, cols, dtype, pad, shift)
            new = torch.full((states, cols), 7.0, device="cuda")
            bad = no_bad()
            d_slots = None if kind == "none" else torch.from_numpy(slots).cuda()
            form = "free" if free else "coupled"
            dmt.dmt_gated_scan_step(gate, value, state, new, h, d_slots, form, bad)
            assert torch.equal(state, kept)
            ref_h, ref_new, off_h = np.zeros((rows, cols)), np.full((states, cols), 7.0), np.zeros((rows, cols))
            f, rest = hs.sigmoid(f64(gate))
            u = f64(value) if free else rest * f64(value)
            for i, s in enumerate(slots):
                if 0 <= s < states and i not in refused:
                    ref_h[i] = ref_new[s] = f[i] * start[s] + u[i]
                    off_h[i] = 12 * U32 * (f[i] * np.abs(start[s]) + np.abs(u[i]))
            off_new = np.zeros((states, cols))
            for i, s in enumerate(slots):
                if 0 <= s < states and i not in refused:
                    off_new[s] = off_h[i] + 1e-37
            close(h, ref_h, U[dtype] * (np.abs(ref_h) + off_h) + off_h + TINY[dtype], "h")
            close(new, ref_new, off_new, "states")
            untouched(around)
            assert int(bad.cpu()) == (refused[0] if refused else -1)
            dmt.dmt_gated_scan_step(gate, value, kept, kept, h, d_slots, form)                # in place
            named = new != 7.0
            assert torch.equal(kept[named], new[named]) and torch.equal(kept[~named], state[~named])


def test_steps_are_the_scan(dmt):
    """A state carried row by row ends where the scan over the rows does."""
    rows, cols = 37, 48
    rng = np.random.default_rng(5)
    gate, value = matrix(rng, 2 * rows, cols, "f32"), matrix(rng, 2 * rows, cols, "f32")
    h, final = torch.empty(2 * rows, cols, device="cuda"), torch.empty(2, cols, device="cuda")
    ws = bytes_buf(dmt.dmt_gated_scan_workspace_bytes(2 * rows, cols))
    dmt.dmt_gated_scan_fwd(gate, value, h, ws, sequences=2, final=final)
    state, out = torch.zeros(2, cols, device="cuda"), torch.empty(2, cols, device="cuda")
    size = float(value.abs().max())
    for t in range(rows):
        dmt.dmt_gated_scan_step(gate[t::rows].contiguous(), value[t::rows].contiguous(), state, state, out)
        # coupled: a mean of values, so sums stay below the largest; 2 x (12 roundings a step, each shrinking, at most 37 of them)
        assert float((out - h[t::rows]).abs().max()) <= 2 * 12 * rows * U32 * size
    assert torch.equal(state, out)


@pytest.mark.parametrize("rows,sequences", [(0, 0), (0, 3), (1, 1), (1000, 7), (5000, 5000), (300_000, 1), (70_000, 3)])
def test_sequence_rows(dmt, rows, sequences):
    rng = np.random.default_rng(rows)
    off = np.concatenate([[0], np.cumsum(lengths_of(rng, rows, sequences))]) if sequences else np.zeros(1, np.int64)
    if rows > 500:                            # rows of none in front and behind
        off = np.maximum(off, 3)
        off[-1] -= 5
        off = np.minimum(off, off[-1])
    out, bad = torch.full((rows,), 99, dtype=torch.int32, device="cuda"), no_bad()
    dmt.dmt_sequence_rows(torch.from_numpy(off.astype(np.int64)).cuda(), out, bad)
    assert np.array_equal(out.cpu().numpy(), hs.sequence_rows(off, rows)) and int(bad.cpu()) == -1


def test_sequence_rows_reports_offsets_that_fall(dmt):
    out, bad = torch.empty(50, dtype=torch.int32, device="cuda"), no_bad()
    dmt.dmt_sequence_rows(torch.tensor([0, 10, 5, 60, -3], device="cuda"), out, bad)
    assert int(bad.cpu()) == 1 and int(out.min()) >= -1 and int(out.max()) < 4


# ------------------------------------------------------------------ dropout

@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (3, 7, 1, 1), (5, 8, 0, 0), (77, 1001, 0, 0), (300, 33, 3, 1), (1000, 256, 0, 0),
                                                 (2, 40_001, 1, 0), (4099, 12, 4, 2)])
def test_dropout(dmt, rows, cols, pad, shift, dtype):
    rng = np.random.default_rng(rows + cols)
    for p, site, seed, step in ((0.1, 0, 1, 0), (0.5, 2047, -3, 2 ** 40 + 5), (0.0, 5, 2 ** 62, -1), (1.0, 1, 9, 9), (1e-6, 3, 9, 9)):
        x, res = matrix(rng, rows, cols, dtype, pad, shift), matrix(rng, rows, cols, dtype, pad + 1, shift)
        state = torch.tensor([seed, step], device="cuda")
        keep = hs.dropout_keep(rows, cols, p, seed, step, site)
        m = hs.dropout_threshold(p)
        scale = 65536 / (65536 - m) if m < 65536 else 0.0
        x[torch.from_numpy(~keep).cuda()] = float("nan")                      # what is left out may hold anything
        kept = np.where(keep, np.nan_to_num(f64(x)), 0.0) * scale
        for residual in (None, res):
            y, around = blank(rows, cols, dtype, pad, shift)
            dmt.dmt_dropout_fwd(x, p, state, y, residual=residual, site=site)
            base = 0.0 if residual is None else f64(residual)
            ref = kept + base
            # the scale, its product and the sum, each one rounding; then the type's
            off = U32 * (2 * np.abs(kept) + np.abs(ref) * (residual is not None)) * 1.01
            close(y, ref, U[dtype] * (np.abs(ref) + off) + off + TINY[dtype], "y")
            untouched(around)
        dx, around = blank(rows, cols, dtype, pad, shift)
        dmt.dmt_dropout_bwd(x, p, state, dx, site=site)
        y, _ = blank(rows, cols, dtype, pad, shift)
        dmt.dmt_dropout_fwd(x, p, state, y, site=site)
        assert torch.equal(dx.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))
        untouched(around)
        dmt.dmt_dropout_bwd(x, p, state, x, site=site)                        # in place
        assert torch.equal(dx, x)
        dmt.dmt_dropout_fwd(y, 0.0, state, y, residual=y)
        assert torch.equal(y, (dx.float() * 2).to(dx.dtype))


def test_dropout_mask_is_the_same_for_every_type_and_stride(dmt):
    state = torch.tensor([11, 22], device="cuda")
    masks = []
    for dtype in ("f32", "f16", "bf16"):
        for pad in (0, 5):
            x = torch.ones(200, 70 + pad, dtype=DT[dtype], device="cuda")[:, :70]
            y = torch.empty(200, 70, dtype=DT[dtype], device="cuda")
            dmt.dmt_dropout_bwd(x, 0.3, state, y, site=4)
            masks.append(y != 0)
    assert all(torch.equal(masks[0], m) for m in masks)
    y2 = torch.empty(200, 70, dtype=torch.bfloat16, device="cuda")
    state[1] += 1
    dmt.dmt_dropout_bwd(torch.ones_like(y2), 0.3, state, y2, site=4)
    assert not torch.equal(y2 != 0, masks[0])


# ------------------------------------------------------------------ rows by expert

def choices(rng, n, k, E, kind):
    e = rng.integers(0, E, (n, k))
    if kind == "skew":
        e = np.minimum(E - 1, (E * rng.random((n, k)) ** 3).astype(np.int64))
    elif kind == "one":
        e[:] = E - 1
    elif kind == "none":
        e[:] = -1
    elif kind == "holes":
        e[rng.random((n, k)) < 0.3] = -2
        e[rng.random((n, k)) < 0.05] = E
        e[rng.random((n, k)) < 0.02] = np.iinfo(np.int32).max
        e[rng.random((n, k)) < 0.02] = np.iinfo(np.int32).min
    return e.astype(np.int32)


def sort_on_gpu(dmt, experts, E, capacity):
    n, k = experts.shape
    i32 = lambda *shape: torch.full(shape, 99, dtype=torch.int32, device="cuda")
    slot, source = i32(n, k), i32(E * capacity if capacity else n * k)
    offsets, counts, bad = i32(E + 1), i32(E), no_bad()
    need = dmt.dmt_expert_sort_workspace_bytes(n, k, E)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda") if need else None
    dmt.dmt_expert_sort(torch.from_numpy(experts).cuda(), E, slot, source, offsets, counts, ws, capacity, bad)
    return slot, source, offsets, counts, bad


@pytest.mark.parametrize("kind", ["uniform", "skew", "one", "none", "holes"])
@pytest.mark.parametrize("n,k,E", [(0, 2, 4), (1, 1, 1), (3, 2, 5), (64, 2, 8), (1000, 3, 7), (2048, 2, 64), (2049, 2, 64), (5000, 1, 1024),
                                   (9000, 4, 60), (40_000, 2, 300), (300_000, 1, 33)])
def test_expert_sort(dmt, n, k, E, kind):
    rng = np.random.default_rng(n + k + E)
    experts = choices(rng, n, k, E, kind)
    for capacity in (0, 1, max(1, n * k // E)):
        got = sort_on_gpu(dmt, experts, E, capacity)
        ref = hs.expert_sort(experts, E, capacity)
        for name, g, r in zip(("slot", "source", "offsets", "counts"), got, ref):
            assert np.array_equal(g.cpu().numpy(), r), (name, capacity)
        over = np.nonzero(experts.reshape(-1) >= E)[0]
        assert int(got[4].cpu()) == (over[0] if len(over) else -1)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,k,E,cols,pad,shift", [(1, 1, 1, 1, 0, 0), (5, 2, 3, 7, 1, 1), (64, 2, 8, 256, 0, 0), (333, 3, 10, 33, 3, 1),
                                                  (700, 4, 16, 1030, 2, 1), (1000, 1, 64, 64, 0, 0), (40, 8, 8, 4099, 1, 0),
                                                  (20, 70, 9, 24, 0, 0)])
def test_expert_moves(dmt, n, k, E, cols, pad, shift, dtype):
    rng = np.random.default_rng(n + cols)
    for kind, capacity in (("uniform", 0), ("holes", 0), ("skew", max(1, n * k // E)), ("none", 3)):
        experts = choices(rng, n, k, E, kind)
        slot, source, _, _, _ = sort_on_gpu(dmt, experts, E, capacity)
        s, src = slot.cpu().numpy(), source.cpu().numpy()
        rows = len(src)
        full, token = src >= 0, np.maximum(src, 0) // k
        x = matrix(rng, n, cols, dtype, pad, shift)
        out, around = blank(rows, cols, dtype, pad, shift)
        dmt.dmt_expert_gather(x, slot, source, out)
        want = np.where(full[:, None], f64(x)[token], 0.0)
        assert np.array_equal(f64(out), want)
        untouched(around)

        z = matrix(rng, rows, cols, dtype, pad, shift)
        z[torch.from_numpy(~full).cuda()] = float("nan")                      # rows that nobody sent anything
        w = torch.from_numpy(rng.random((n, k)).astype(np.float32)).cuda()
        z64, w64 = np.nan_to_num(f64(z)), np.where(s >= 0, f64(w), 0.0)
        for weights in (w, None):
            ww = w64 if weights is not None else (s >= 0).astype(np.float64)
            terms = ww[:, :, None] * z64[np.maximum(s, 0)] if rows else np.zeros((n, k, cols))
            ref, size = terms.sum(1), np.abs(terms).sum(1)
            for yd in sorted({dtype, "f32", "bf16"}):
                y, around = blank(n, cols, yd, pad, shift)
                dmt.dmt_expert_combine(z, slot, weights, y)
                off = (k + 1) * U32 * size
                close(y, ref, U[yd] * (np.abs(ref) + off) + off + TINY[yd], "y")
                untouched(around)
        for gd in sorted({dtype, "f32"}):
            dy = matrix(rng, n, cols, gd, pad, shift)
            for weights in (w, None):
                ww = w64 if weights is not None else (s >= 0).astype(np.float64)
                dz, around = blank(rows, cols, gd, pad, shift)
                dw = torch.full((n, k), 7.0, device="cuda")
                dmt.dmt_expert_combine_bwd(dy, z, slot, source, weights, dz, dw)
                dy64 = f64(dy)
                ref = np.where(full[:, None], dy64[token] * ww.reshape(-1)[np.maximum(src, 0)][:, None], 0.0) if rows else np.zeros((0, cols))
                close(dz, ref, (U[gd] + 2 * U32) * np.abs(ref) + TINY[gd], "dz")
                untouched(around)
                terms = dy64[:, None, :] * z64[np.maximum(s, 0)] * (s >= 0)[:, :, None] if rows else np.zeros((n, k, cols))
                # a lane's running sum of cols / 64 + 8 terms, then six sums over lanes
                close(dw, terms.sum(2), (cols / 64 + 16) * U32 * np.abs(terms).sum(2) + 1e-37, "dweights")
                only, only_w = torch.full_like(dz, 7.0), torch.full_like(dw, 7.0)
                dmt.dmt_expert_combine_bwd(dy, None, slot, source, weights, only)
                dmt.dmt_expert_combine_bwd(dy, z, slot, None, weights, None, only_w)
                assert torch.equal(only, dz) and torch.equal(only_w, dw)


def test_rows_and_tokens_past_32_bits(dmt):
    """Strides whose offsets pass 2^32 elements."""
    free = torch.cuda.mem_get_info()[0]
    if free < 40 << 30:
        pytest.skip("40 GiB of GPU memory needed")
    rows, cols, stride = 70, 24, (1 << 32) // 64
    big = torch.zeros(rows * stride, dtype=torch.bfloat16, device="cuda")
    x = big.view(rows, stride)[:, :cols]
    rng = np.random.default_rng(1)
    x.copy_(torch.from_numpy(rng.normal(size=(rows, cols))))
    state = torch.tensor([1, 2], device="cuda")
    far = big.view(rows, stride)[:, cols:2 * cols]
    near = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    small = x.contiguous()
    for a, b in ((x, small),):
        dmt.dmt_dropout_bwd(a, 0.4, state, far)
        dmt.dmt_dropout_bwd(b, 0.4, state, near)
        assert torch.equal(far, near)
        ws = bytes_buf(dmt.dmt_gated_scan_workspace_bytes(rows, cols))
        dmt.dmt_gated_scan_fwd(a, a, far, ws)
        dmt.dmt_gated_scan_fwd(b, b, near, ws)
        assert torch.equal(far, near)
        slot = torch.arange(rows, dtype=torch.int32, device="cuda").flip(0)[:, None].contiguous()
        source = slot[:, 0].contiguous()
        dmt.dmt_expert_gather(a, slot, source, far)
        assert torch.equal(far, small.flip(0))
        dmt.dmt_expert_combine(far, slot, None, near)
        assert torch.equal(near, small)


# ------------------------------------------------------------------ nothing, streams, graphs

def test_calls_of_nothing(dmt):
    f32 = lambda *shape: torch.full(shape, 7.0, device="cuda")
    i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")
    x, state, rng = f32(0, 24), f32(3, 24), torch.zeros(2, dtype=torch.int64, device="cuda")
    for seq, n in ((i32(0), 3), (None, 0), (None, 3)):
        final, dinitial = f32(n, 24), f32(n, 24)
        dmt.dmt_gated_scan_fwd(x, x, x, None, sequence_of=seq, sequences=n, final=final)
        dmt.dmt_gated_scan_bwd(x, x, x, x, x, None, None, sequence_of=seq, sequences=n, dinitial=dinitial)
        assert bool((final == 7).all()) and bool((dinitial == 7).all())       # sequences without rows are left as they were
    dmt.dmt_gated_scan_step(x, x, state, state, x, i32(0))
    dmt.dmt_dropout_fwd(x, 0.5, rng, x)
    dmt.dmt_dropout_bwd(x, 0.5, rng, x)
    slot, source = i32(0, 2), torch.full((12,), 9, dtype=torch.int32, device="cuda")
    offsets, counts = i32(5) + 9, i32(4) + 9
    dmt.dmt_expert_sort(i32(0, 2), 4, slot, source, offsets, counts, None, capacity=3)
    assert source.tolist() == [-1] * 12 and offsets.tolist() == [0, 3, 6, 9, 12] and counts.tolist() == [0] * 4
    out = f32(12, 24)
    dmt.dmt_expert_gather(x, slot, source, out)                               # no tokens: every row is empty
    assert bool((out == 0).all())
    out = f32(12, 24)
    dmt.dmt_expert_combine(out, slot, None, x)
    dmt.dmt_expert_combine_bwd(x, None, slot, source, None, out)
    assert bool((out == 0).all())
    y, none = f32(5, 24), i32(0)
    dmt.dmt_expert_combine(x, torch.full((5, 2), -1, dtype=torch.int32, device="cuda"), None, y)      # no rows: sums of nothing
    assert bool((y == 0).all()) and none.numel() == 0
    # only rows of no sequence
    h, final = f32(20, 24), f32(2, 24)
    ws = bytes_buf(dmt.dmt_gated_scan_workspace_bytes(20, 24))
    dmt.dmt_gated_scan_fwd(f32(20, 24) / 0, f32(20, 24) / 0, h, ws, sequence_of=i32(20) - 1, sequences=2, final=final)
    assert bool((h == 0).all()) and bool((final == 7).all())


def _block(dmt, seed):
    """State of a small chain of all operators; run(s) goes through it once."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n, C, E, k, cap = 700, 72, 6, 2, 200
    rnd = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    f32 = lambda *shape: torch.zeros(*shape, device="cuda")
    i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")
    s = dict(n=n, C=C, E=E, cap=cap, gate=rnd(n, C) * 2, value=rnd(n, C), off=torch.tensor([0, 5, 5, 300, 690], device="cuda"),
             seq=i32(n), h=f32(n, C), final=f32(4, C), r=f32(n, C), rng=torch.tensor([seed, 0], device="cuda"),
             experts=torch.randint(-1, E, (n, k), generator=g, device="cuda", dtype=torch.int32), slot=i32(n, k), source=i32(E * cap),
             offsets=i32(E + 1), counts=i32(E), rows=f32(E * cap, C), w=rnd(n, k), y=f32(n, C), dz=f32(E * cap, C), dw=f32(n, k),
             dx=f32(n, C), dh=f32(n, C), dg=f32(n, C), dv=f32(n, C), state=rnd(50, C), slots=torch.randperm(50, generator=g, device="cuda")[:20]
             .to(torch.int32), new=f32(50, C), hs=f32(20, C),
             kept=bytes_buf(dmt.dmt_gated_scan_kept_bytes(n, C)), ws=bytes_buf(max(dmt.dmt_gated_scan_workspace_bytes(n, C),
                                                                                  dmt.dmt_expert_sort_workspace_bytes(n, k, E))))
    return s


def _run_block(dmt, s, stream=None):
    kw = dict(stream=stream)
    dmt.dmt_sequence_rows(s["off"], s["seq"], **kw)
    dmt.dmt_gated_scan_fwd(s["gate"], s["value"], s["h"], s["ws"], sequence_of=s["seq"], sequences=4, final=s["final"], kept=s["kept"], **kw)
    dmt.dmt_dropout_fwd(s["h"], 0.3, s["rng"], s["r"], residual=s["value"], site=2, **kw)
    dmt.dmt_expert_sort(s["experts"], s["E"], s["slot"], s["source"], s["offsets"], s["counts"], s["ws"], s["cap"], **kw)
    dmt.dmt_expert_gather(s["r"], s["slot"], s["source"], s["rows"], **kw)
    dmt.dmt_expert_combine(s["rows"], s["slot"], s["w"], s["y"], **kw)
    dmt.dmt_expert_combine_bwd(s["y"], s["rows"], s["slot"], s["source"], s["w"], s["dz"], s["dw"], **kw)
    dmt.dmt_expert_combine(s["dz"], s["slot"], None, s["dx"], **kw)
    dmt.dmt_dropout_bwd(s["dx"], 0.3, s["rng"], s["dh"], site=2, **kw)
    dmt.dmt_gated_scan_bwd(s["gate"], s["value"], s["dh"], s["dg"], s["dv"], s["kept"], s["ws"], sequence_of=s["seq"], sequences=4, **kw)
    dmt.dmt_gated_scan_step(s["gate"][:20], s["value"][:20], s["state"], s["new"], s["hs"], s["slots"], **kw)


OUT = ["seq", "h", "final", "r", "slot", "source", "offsets", "counts", "rows", "y", "dz", "dw", "dx", "dh", "dg", "dv", "new", "hs"]


def _cleared(s):
    for o in OUT:
        s[o].fill_(-5)


def test_another_stream_and_graphs_that_share_a_workspace_give_the_same(dmt):
    a, b = _block(dmt, 1), _block(dmt, 2)
    b["ws"] = a["ws"]                                       # ordered by the caller: one after another
    eager = []
    for s in (a, b):
        _cleared(s)                                         # (rows that no call writes stay so)
        _run_block(dmt, s)
        eager.append({o: s[o].clone() for o in OUT})
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    _cleared(a)
    side.wait_stream(torch.cuda.current_stream())
    _run_block(dmt, a, side)
    torch.cuda.synchronize()
    assert all(torch.equal(a[o], eager[0][o]) for o in OUT)
    graphs = []
    for s in (a, b):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _run_block(dmt, s)
        graphs.append(graph)
    for turn in range(4):
        for i, s in ((0, a), (1, b)) if turn % 2 == 0 else ((1, b), (0, a)):
            _cleared(s)
            if turn == 3:                                   # the replay reads what the tensors hold now: other masks
                s["rng"][1] = 5
            graphs[i].replay()
            torch.cuda.synchronize()
            if turn < 3:
                assert all(torch.equal(s[o], eager[i][o]) for o in OUT), (turn, i)
            else:
                by_graph = {o: s[o].clone() for o in OUT}
                assert not torch.equal(by_graph["r"], eager[i]["r"]) and torch.equal(by_graph["h"], eager[i]["h"])
                _cleared(s)
                _run_block(dmt, s)
                assert all(torch.equal(s[o], by_graph[o]) for o in OUT)


def test_step_of_many_rows_with_the_same_slot(dmt):
    rng = np.random.default_rng(8)
    rows, cols, states = 6000, 8, 300_000
    slots = rng.permutation(states)[:rows].astype(np.int32)
    slots[3000:3100] = slots[:100]                           # far behind
    slots[5001] = slots[5000]                                # in one block
    slots[4096 * 1 + 7] = slots[2] + 131072 if slots[2] + 131072 < states else -1      # the same bit, another slot
    slots[200:220] = -4
    first = {}
    want_bad = []
    for i, v in enumerate(slots):
        if v >= 0 and first.setdefault(int(v), i) != i:
            want_bad.append(i)
    gate = torch.full((rows, cols), -100.0, device="cuda")   # shut: the state becomes the value
    value = torch.arange(rows, device="cuda", dtype=torch.float32)[:, None].expand(rows, cols).contiguous()
    state, h, bad = torch.full((states, cols), -7.0, device="cuda"), torch.empty(rows, cols, device="cuda"), no_bad()
    dmt.dmt_gated_scan_step(gate, value, state, state, h, torch.from_numpy(slots).cuda(), first_bad=bad)
    assert int(bad.cpu()) == want_bad[0]
    want = np.full(states, -7.0)
    for v, i in first.items():
        want[v] = i
    assert np.allclose(state[:, 0].cpu().numpy(), want, rtol=0, atol=1e-30)
    refused = np.isin(np.arange(rows), want_bad) | (slots < 0)
    assert np.array_equal(h[:, 3].cpu().numpy() == 0, refused | (np.arange(rows) == 0))


def test_tensors_that_are_refused(dmt):
    x = torch.ones(4, 8, device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    ws, rng = bytes_buf(1 << 16), torch.zeros(2, dtype=torch.int64, device="cuda")
    calls = [lambda: dmt.dmt_gated_scan_fwd(x, x.cpu(), x, ws), lambda: dmt.dmt_gated_scan_fwd(x, x[:, :7], x, ws),
             lambda: dmt.dmt_gated_scan_fwd(x, x.half(), x, ws), lambda: dmt.dmt_gated_scan_fwd(x, x, x, ws.cpu()),
             lambda: dmt.dmt_gated_scan_fwd(x, x, x, ws, sequence_of=ids.long(), sequences=1),
             lambda: dmt.dmt_gated_scan_fwd(x, x, x, ws, initial=x), lambda: dmt.dmt_gated_scan_fwd(x, x.t().contiguous().t(), x, ws),
             lambda: dmt.dmt_gated_scan_step(x, x, x, x[:3], x, ids), lambda: dmt.dmt_gated_scan_step(x, x, x.half(), x, x, ids),
             lambda: dmt.dmt_dropout_fwd(x, 0.5, rng.cpu(), x), lambda: dmt.dmt_dropout_fwd(x, 0.5, rng[:1], x),
             lambda: dmt.dmt_dropout_fwd(x, 0.5, rng, x, residual=x.half()), lambda: dmt.dmt_dropout_bwd(x, 0.5, rng, x.half()),
             lambda: dmt.dmt_expert_gather(x, ids[:, None], ids[:3], x), lambda: dmt.dmt_expert_gather(x.half(), ids[:, None], ids, x),
             lambda: dmt.dmt_expert_combine(x, ids[:, None].long(), None, x),
             lambda: dmt.dmt_expert_combine(x, ids[:, None], x, x),
             lambda: dmt.dmt_expert_sort(ids[:, None], 3, ids[:, None], ids[:3], None, None, ws)]
    for i, c in enumerate(calls):
        with pytest.raises(AssertionError):
            c()
            raise ValueError("call %d was taken" % i)
    for c in (lambda: dmt.dmt_gated_scan_fwd(x, x, x, ws, form="other"),):
        with pytest.raises(KeyError):
            c()
