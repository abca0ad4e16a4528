"""The gated recurrence where exp(-gate) runs out of float32: finite gates whose sigmoid, or whose sigmoid's complement, is below 2^-126.

A value below 2^-126 may be taken as 0, so f and 1 - f may each be off by FLUSH = 2^-126 besides what oracle/history.py counts: a state by FLUSH
times the states and values that each of its rows multiplies, a gradient by FLUSH times the products that they are factors of.
"""
import numpy as np
import pytest
import torch

from oracle import history as hs
from test_gpu_sequence import DT, TINY, U, U32, bytes_buf, close, f64, matrix

pytestmark = pytest.mark.gpu

FLUSH = 2.0 ** -126
# exp(87.34) passes 2^126, exp(88.72) the largest float32, exp(-87.34) goes below 2^-126; 16.6 and 17.4 are where 1 - f comes to 1
EDGES = [87.0, 87.25, 87.3, 87.34, 87.5, 88.0, 88.5, 88.7, 88.72, 88.73, 89.0, 104.0, 16.6, 17.4, 30.0]


@pytest.fixture(scope="module")
def dmt():
    import paper_2403_00877_amd as d
    return d


def edge_gates(gate, rng):
    """Every third row and every fifth column of the others: gates from EDGES, of either sign."""
    rows, cols = gate.shape
    edge = torch.tensor([s * e for e in EDGES for s in (-1.0, 1.0)], dtype=gate.dtype, device="cuda")
    put = torch.zeros(rows, cols, dtype=torch.bool, device="cuda")
    put[::3] = True
    put[:, ::5] = True
    pick = torch.from_numpy(rng.integers(0, len(edge), (rows, cols))).cuda()
    gate.copy_(torch.where(put, edge[pick], gate))


@pytest.mark.parametrize("dtype,gd", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("free", [False, True])
@pytest.mark.parametrize("rows,cols,sequences,ragged", [(60, 37, 2, False), (1, 30, 1, False), (1600, 5, 100, False), (3000, 65, 3, True),
                                                        (2500, 270, 40, True), (9000, 33, 9, False)])
def test_gates_at_the_ends_of_exp(dmt, rows, cols, sequences, ragged, free, dtype, gd):
    rng = np.random.default_rng(rows + cols)
    gate, value, dh = matrix(rng, rows, cols, dtype, 1, 1, 3.0, 1.0), matrix(rng, rows, cols, dtype, 3), matrix(rng, rows, cols, gd)
    edge_gates(gate, rng)
    seq = np.sort(rng.integers(0, sequences, rows)).astype(np.int32) if ragged else None
    initial, dfinal = (torch.from_numpy(rng.normal(size=(sequences, cols)).astype(np.float32)).cuda() for _ in range(2))
    h, dgate, dvalue = torch.empty(rows, cols, dtype=DT[dtype], device="cuda"), torch.empty_like(dh), torch.empty_like(dh)
    final, dinitial = torch.full((sequences, cols), 7.0, device="cuda"), torch.full((sequences, cols), 7.0, device="cuda")
    kept, ws = bytes_buf(dmt.dmt_gated_scan_kept_bytes(rows, cols)), bytes_buf(dmt.dmt_gated_scan_workspace_bytes(rows, cols))
    where = dict(form="free" if free else "coupled", sequence_of=None if seq is None else torch.from_numpy(seq).cuda(), sequences=sequences,
                 initial=initial)
    dmt.dmt_gated_scan_fwd(gate, value, h, ws, final=final, kept=kept, **where)
    dmt.dmt_gated_scan_bwd(gate, value, dh, dgate, dvalue, kept, ws, dfinal=dfinal, dinitial=dinitial, **where)
    found = hs.runs(seq, rows, sequences)
    seven = np.full((sequences, cols), 7.0)
    ref = hs.scan_fwd(f64(gate), f64(value), free, found, f64(initial), seven)
    back = hs.scan_bwd(ref, f64(value), free, found, f64(dh), f64(dfinal), seven)
    # a state is a sum over the rows before it of at most |h| + |value| each, an l over the rows behind it of |l|
    most = max(float(np.abs(x).max()) for x in (ref["h"], ref["prev"], f64(value)))
    most_l = float(np.abs(f64(dh)).max() + np.abs(f64(dfinal)).max()) * rows
    flush = 2 * rows * FLUSH * most
    close(h, ref["h"], U[dtype] * (np.abs(ref["h"]) + ref["off"]) + ref["off"] + flush + TINY[dtype], "h")
    close(final, ref["final"], ref["final_off"] + flush, "final")
    for name, got, more in (("dgate", dgate, 4 * most_l * most * FLUSH), ("dvalue", dvalue, 2 * most_l * FLUSH)):
        off = back[name + "_off"]
        close(got, back[name], U[gd] * (np.abs(back[name]) + off) + off + more + TINY[gd], name)
    close(dinitial, back["dinitial"], back["dinitial_off"] + 2 * most_l * FLUSH, "dinitial")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("free", [False, True])
@pytest.mark.parametrize("rows,cols,states,slots", [(1, 30, 1, False), (60, 37, 90, True), (1500, 33, 1600, True), (700, 64, 700, False)])
def test_step_with_gates_at_the_ends_of_exp(dmt, rows, cols, states, slots, free, dtype):
    rng = np.random.default_rng(rows + cols)
    gate, value = matrix(rng, rows, cols, dtype, 1, 1, 3.0), matrix(rng, rows, cols, dtype)
    edge_gates(gate, rng)
    at = rng.permutation(states)[:rows].astype(np.int32) if slots else np.arange(rows, dtype=np.int32)
    state = torch.from_numpy(rng.normal(size=(states, cols)).astype(np.float32)).cuda()
    new, h = torch.full((states, cols), 7.0, device="cuda"), torch.empty(rows, cols, dtype=DT[dtype], device="cuda")
    dmt.dmt_gated_scan_step(gate, value, state, new, h, torch.from_numpy(at).cuda() if slots else None, "free" if free else "coupled")
    f, rest = hs.sigmoid(f64(gate))
    u = f64(value) if free else rest * f64(value)
    before, want = f64(state)[at], np.full((states, cols), 7.0)
    ref = f * before + u
    want[at] = ref
    # the roundings and the exponential's argument as oracle/history.py counts them
    off = 12 * U32 * (f * np.abs(before) + np.abs(u)) + 1.25 * U32 * np.abs(f64(gate)) * f * rest * (np.abs(before) + np.abs(f64(value)))
    off = off + FLUSH * (np.abs(before) + np.abs(f64(value))) + 1e-37
    close(h, ref, U[dtype] * (np.abs(ref) + off) + off + TINY[dtype], "h")
    off_new = np.zeros((states, cols))
    off_new[at] = off
    close(new, want, off_new, "states")
