"""NaN and infinities in the gated recurrence: where they must be seen, and where they must not be."""
import numpy as np
import pytest
import torch

from oracle import history as hs
from test_gpu_sequence import TINY, U, bytes_buf, f64, matrix

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dmt():
    import paper_2403_00877_amd as d
    return d


def same_or_lost(got, ref, tol, what):
    """Near the reference where it is finite, NaN where it is NaN, no finite number where it is infinite (a stretch's product of f that ran
    out of float32 makes NaN of an infinity)."""
    got = f64(got)
    finite, nan = np.isfinite(ref), np.isnan(ref)
    with np.errstate(invalid="ignore"):
        wrong = np.where(finite, ~(np.abs(got - ref) <= tol), np.where(nan, ~np.isnan(got), np.isfinite(got)))
    if wrong.any():
        at = np.unravel_index(int(np.argmax(wrong)), wrong.shape)
        raise AssertionError("%s: %d of %d off, first at %s: %r, %r expected" % (what, int(wrong.sum()), wrong.size, at, got[at], ref[at]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("free", [False, True])
@pytest.mark.parametrize("rows,cols,sequences,dense", [(40, 5, 2, True), (900, 40, 9, False), (2400, 33, 300, True)])
def test_gradients_of_a_nan(dmt, rows, cols, sequences, dense, free, dtype):
    """A NaN gate makes NaN of its own row's gradients (free: dvalue = l does not depend on f) and of the rows before it; a NaN value of its
    row's dgate and of the dgate of the rows behind it."""
    rng = np.random.default_rng(rows)
    gate, value, dh = (matrix(rng, rows, cols, dtype) for _ in range(3))
    per = rows // sequences
    gate[per // 2, 1] = value[per + per // 3, 2] = gate[rows - 1, 0] = gate[per, 3] = dh[per // 2, 4] = float("nan")
    seq = None if dense else np.repeat(np.arange(sequences), per).astype(np.int32)
    h, dgate, dvalue = (torch.empty_like(gate) for _ in range(3))
    kept, ws = bytes_buf(dmt.dmt_gated_scan_kept_bytes(rows, cols)), bytes_buf(dmt.dmt_gated_scan_workspace_bytes(rows, cols))
    where = dict(form="free" if free else "coupled", sequence_of=None if dense else torch.from_numpy(seq).cuda(), sequences=sequences)
    dmt.dmt_gated_scan_fwd(gate, value, h, ws, kept=kept, **where)
    dmt.dmt_gated_scan_bwd(gate, value, dh, dgate, dvalue, kept, ws, **where)
    found = hs.runs(seq, rows, sequences)
    ref = hs.scan_fwd(f64(gate), f64(value), free, found)
    back = hs.scan_bwd(ref, f64(value), free, found, f64(dh))
    if not free:
        assert np.isnan(back["dvalue"][per // 2, 1]) and np.isnan(back["dvalue"][rows - 1, 0])
    same_or_lost(h, ref["h"], U[dtype] * (np.abs(ref["h"]) + ref["off"]) + ref["off"] + TINY[dtype], "h")
    for name, got in (("dgate", dgate), ("dvalue", dvalue)):
        off = back[name + "_off"]
        same_or_lost(got, back[name], U[dtype] * (np.abs(back[name]) + off) + off + TINY[dtype], name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("free", [False, True])
@pytest.mark.parametrize("lengths,cols", [([700, 3000, 40, 2000, 3260], 40), ([3000, 3000, 3000], 40), ([900, 1500, 10, 20, 1570], 140)])
def test_what_is_lost_stays_in_its_sequence_across_chunks(dmt, lengths, cols, free, dtype):
    """Sequences of several chunks of rows, two of them with NaN and infinities in rows, states and gradients."""
    rows, n = sum(lengths), len(lengths)
    begin = np.concatenate([[0], np.cumsum(lengths)])
    rng = np.random.default_rng(rows + cols)
    gate, value = matrix(rng, rows, cols, dtype, scale=2.0, mean=1.0), matrix(rng, rows, cols, dtype)
    dh = matrix(rng, rows, cols, dtype)
    initial, dfinal = (torch.from_numpy(rng.normal(size=(n, cols)).astype(np.float32)).cuda() for _ in range(2))
    dense = len(set(lengths)) == 1
    seq = None if dense else np.repeat(np.arange(n), lengths).astype(np.int32)
    where = dict(form="free" if free else "coupled", sequence_of=None if dense else torch.from_numpy(seq).cuda(), sequences=n, initial=initial)
    found, outs = hs.runs(seq, rows, n), []
    a, b, e = int(begin[1]), int(begin[2]), int(begin[n - 1])
    for poison in (False, True):
        if poison:
            gate[a + 800, 3], value[a + 200, 4], value[b - 1, 5], dh[a + 1400, 6], dh[b - 3, 7] = (float(x) for x in ("nan", "inf", "nan", "nan", "-inf"))
            initial[1, 8], dfinal[1, 9], initial[n - 1, 10], dfinal[n - 1, 11] = (float(x) for x in ("nan", "inf", "-inf", "nan"))
            gate[e, 12], gate[e, 13] = float("nan"), float("-inf")            # (shut: the state starts anew)
        h, dgate, dvalue = (torch.empty_like(gate) for _ in range(3))
        final, dinitial = (torch.full((n, cols), 7.0, device="cuda") for _ in range(2))
        kept, ws = bytes_buf(dmt.dmt_gated_scan_kept_bytes(rows, cols)), bytes_buf(dmt.dmt_gated_scan_workspace_bytes(rows, cols))
        ws.fill_(0xFF)
        dmt.dmt_gated_scan_fwd(gate, value, h, ws, final=final, kept=kept, **where)
        dmt.dmt_gated_scan_bwd(gate, value, dh, dgate, dvalue, kept, ws, dfinal=dfinal, dinitial=dinitial, **where)
        outs.append((h, dgate, dvalue, final, dinitial))
    in_rows = torch.ones(rows, cols, dtype=torch.bool, device="cuda")
    in_rows[a:b, 3:10], in_rows[e:, 10:14] = False, False
    in_states = torch.ones(n, cols, dtype=torch.bool, device="cuda")
    in_states[1, 3:10], in_states[n - 1, 10:14] = False, False
    for clean, got, which in zip(*outs, (in_rows, in_rows, in_rows, in_states, in_states)):
        assert torch.equal(clean[which], got[which]) and bool(torch.isfinite(got[which]).all())
    seven = np.full((n, cols), 7.0)
    with np.errstate(invalid="ignore"):
        ref = hs.scan_fwd(f64(gate), f64(value), free, found, f64(initial), seven)
        back = hs.scan_bwd(ref, f64(value), free, found, f64(dh), f64(dfinal), seven)
        same_or_lost(h, ref["h"], U[dtype] * (np.abs(ref["h"]) + ref["off"]) + ref["off"] + TINY[dtype], "h")
        same_or_lost(final, ref["final"], ref["final_off"] + 1e-37, "final")
        for name, got in (("dgate", dgate), ("dvalue", dvalue)):
            off = back[name + "_off"]
            same_or_lost(got, back[name], U[dtype] * (np.abs(back[name]) + off) + off + TINY[dtype], name)
        same_or_lost(dinitial, back["dinitial"], back["dinitial_off"] + 1e-37, "dinitial")
