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
