"""The gated recurrence over several hundred chunks of rows with gates that are neither open nor shut; strides past 2^32 elements for what reads
and writes gradients and for the step."""
import numpy as np
import pytest
import torch

from oracle import history as hs
from test_gpu_sequence import DT, TINY, U, bytes_buf, close, f64, matrix

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dmt():
    import paper_2403_00877_amd as d
    return d


@pytest.mark.parametrize("rows,cols,starts,dtype,free", [(80_000, 130, [0], "bf16", False), (80_000, 130, [0, 37, 79_000], "bf16", True),
                                                         (60_000, 33, [0, 20_001, 20_002], "f32", False)])
def test_gated_scan_over_hundreds_of_chunks(dmt, rows, cols, starts, dtype, free):
    """80000 x 130 bfloat16 is cut into 625 chunks of 128 rows.  Gates between 2 and 12: some states are gone after ten rows, some last for
    100000; channel 0 is open and empty, so that a state (a gradient) passes from one end to the other."""
    rng = np.random.default_rng(rows + len(starts))
    n = len(starts)
    gate, value, dh = (matrix(rng, rows, cols, t) for t in (dtype, dtype, dtype))
    gate.add_(torch.linspace(2.0, 12.0, cols, device="cuda").to(gate.dtype))
    gate[:, 0], value[:, 0], dh[:, 0] = 60.0, 0.0, 0.0
    seq = np.zeros(rows, np.int32)
    for s in starts[1:]:
        seq[s:] += 1
    state = lambda: torch.from_numpy((rng.normal(size=(n, cols)) + 4).astype(np.float32)).cuda()
    initial, dfinal = state(), state()
    final, dinitial = (torch.full((n, cols), 7.0, device="cuda") for _ in range(2))
    h, dgate, dvalue = (torch.empty(rows, cols, dtype=DT[dtype], device="cuda") for _ in range(3))
    kept, ws = bytes_buf(dmt.dmt_gated_scan_kept_bytes(rows, cols)), bytes_buf(dmt.dmt_gated_scan_workspace_bytes(rows, cols))
    where = dict(form="free" if free else "coupled", sequence_of=torch.from_numpy(seq).cuda() if n > 1 else None, sequences=n, initial=initial)
    dmt.dmt_gated_scan_fwd(gate, value, h, ws, final=final, kept=kept, **where)
    dmt.dmt_gated_scan_bwd(gate, value, dh, dgate, dvalue, kept, ws, dfinal=dfinal, dinitial=dinitial, **where)
    found = hs.runs(seq if n > 1 else None, rows, n)
    seven = np.full((n, cols), 7.0)
    ref = hs.scan_fwd(f64(gate), f64(value), free, found, f64(initial), seven)
    back = hs.scan_bwd(ref, f64(value), free, found, f64(dh), f64(dfinal), seven)
    assert torch.equal(final[:, 0], initial[:, 0]) and torch.equal(dinitial[:, 0], dfinal[:, 0])
    close(h, ref["h"], U[dtype] * (np.abs(ref["h"]) + ref["off"]) + ref["off"] + TINY[dtype], "h")
    close(final, ref["final"], ref["final_off"] + 1e-37, "final")
    for name, got in (("dgate", dgate), ("dvalue", dvalue)):
        off = back[name + "_off"]
        close(got, back[name], U[dtype] * (np.abs(back[name]) + off) + off + TINY[dtype], name)
    close(dinitial, back["dinitial"], back["dinitial_off"] + 1e-37, "dinitial")


def test_gradients_and_steps_past_32_bits(dmt):
    """Rows 2^26 elements apart."""
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("20 GiB of GPU memory needed")
    rows, cols, stride = 70, 24, 1 << 26
    big = torch.zeros(rows * stride, dtype=torch.bfloat16, device="cuda").view(rows, stride)
    far = [big[:, i * cols:(i + 1) * cols] for i in range(6)]
    rng = np.random.default_rng(2)
    for t in far[:3]:
        t.copy_(torch.from_numpy(rng.normal(size=(rows, cols))))
    near = [t.contiguous() for t in far]
    state = torch.from_numpy(rng.normal(size=(rows, cols)).astype(np.float32)).cuda()
    slots = torch.from_numpy(rng.permutation(rows).astype(np.int32)).cuda()
    experts = torch.from_numpy(rng.integers(0, 3, (rows // 2, 2)).astype(np.int32)).cuda()
    slot, source = torch.empty_like(experts), torch.empty(rows, dtype=torch.int32, device="cuda")
    dmt.dmt_expert_sort(experts, 3, slot, source, None, None, None)
    weights = torch.from_numpy(rng.random((rows // 2, 2)).astype(np.float32)).cuda()
    outs = []
    for gate, value, dh, a, b, c in (near, far):
        kept, ws = bytes_buf(dmt.dmt_gated_scan_kept_bytes(rows, cols)), bytes_buf(dmt.dmt_gated_scan_workspace_bytes(rows, cols))
        dmt.dmt_gated_scan_fwd(gate, value, c, ws, kept=kept, sequences=2)
        dmt.dmt_gated_scan_bwd(gate, value, dh, a, b, kept, ws, sequences=2)
        out = [t.contiguous().clone() for t in (a, b, c)]
        for s in (slots, None):
            new = torch.zeros_like(state)
            dmt.dmt_gated_scan_step(gate, value, state, new, c, s)
            out += [new, c.contiguous().clone()]
        dweights = torch.empty_like(weights)
        dmt.dmt_expert_combine_bwd(dh[:rows // 2], value, slot, source, weights, a, dweights)
        outs.append(out + [a.contiguous().clone(), dweights])
    assert all(torch.equal(x, y) for x, y in zip(*outs)) and all(float(x.float().abs().sum()) > 0 for x in outs[0])


def test_gradients_of_weights_need_the_experts_rows(dmt):
    dy, slot, weights = torch.ones(3, 4, device="cuda"), torch.zeros(3, 2, dtype=torch.int32, device="cuda"), torch.ones(3, 2, device="cuda")
    with pytest.raises(AssertionError, match="dweights"):
        dmt.dmt_expert_combine_bwd(dy, None, slot, None, weights, None, torch.zeros(3, 2, device="cuda"))


def test_ids_need_the_number_of_sequences(dmt):
    x, ids, ws = torch.ones(4, 8, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda"), bytes_buf(256)
    h = torch.zeros(4, 8, device="cuda")
    with pytest.raises(AssertionError, match="sequences"):
        dmt.dmt_gated_scan_fwd(x, x, h, ws, sequence_of=ids)
    dmt.dmt_gated_scan_fwd(x, x, h, ws, sequence_of=ids, sequences=4)
    assert bool((h == h[:1]).all()) and bool((h > 0).all())
