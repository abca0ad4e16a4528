"""More rows than one launch of 2^32 threads holds, and rows of numbers that fill 31 bits."""
import numpy as np
import pytest
import torch

from oracle import history as hs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dmt():
    import paper_2403_00877_amd as d
    return d


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def need(gib):
    free = torch.cuda.mem_get_info()[0]
    if free < gib << 30:
        pytest.skip("%d GiB of GPU memory needed, %.0f are free" % (gib, free / 2 ** 30))


def test_dropout_of_more_rows_than_a_launch_holds(dmt):
    """Two groups of eight a row and 2^31 - 1 rows, in place."""
    need(60)
    rows, cols = (1 << 31) - 1, 9
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    state = torch.tensor([5, 6], device="cuda")
    dmt.dmt_dropout_bwd(x, 0.25, state, x, site=9)
    for a in (0, (1 << 31) - 1 - 300, (1 << 30) - 150, 12_345_678):
        part = x[a:a + 300].float().cpu().numpy()
        groups = np.arange(2, dtype=np.uint64) + np.uint64(9 << 21)
        row = np.arange(a, a + 300, dtype=np.uint64)[:, None]
        words = hs.philox([np.broadcast_to(groups, (300, 2)), np.broadcast_to(row, (300, 2)), np.uint64(6), np.uint64(0)], [5, 0])
        half = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=2).reshape(300, 16)[:, :cols]
        keep = half >= np.uint64(hs.dropout_threshold(0.25))
        assert np.array_equal(part != 0, keep), a
    share = sum(float((x[a:a + (1 << 24)] != 0).float().mean()) for a in range(0, rows, 1 << 28)) / 8
    assert abs(share - 0.75) < 1e-3


def test_steps_and_moves_of_narrow_rows(dmt):
    """2^26 rows of one element, and experts' rows of one."""
    need(8)
    rows = (1 << 26) + 3
    gate = torch.full((rows, 1), -100.0, dtype=torch.bfloat16, device="cuda")
    value = (torch.arange(rows, device="cuda") % 251).to(torch.bfloat16)[:, None]
    state, h = torch.full((rows, 1), 3.0, device="cuda"), torch.empty_like(value)
    dmt.dmt_gated_scan_step(gate, value, state, state, h)
    assert torch.equal(h, value) and torch.equal(state, value.float())
    slot = torch.arange(rows, device="cuda", dtype=torch.int32).flip(0)[:, None].contiguous()
    out = torch.empty_like(value)
    dmt.dmt_expert_gather(value, slot, slot[:, 0].contiguous(), out)
    assert torch.equal(out, value.flip(0))
    back = torch.empty_like(value)
    dmt.dmt_expert_combine(out, slot, None, back)
    assert torch.equal(back, value)


def test_scan_of_very_many_rows(dmt):
    """2^27 rows of two channels, 33 sequences: sums of ones that start again."""
    need(16)
    rows, cols = 1 << 27, 2
    starts = torch.arange(33, device="cuda") * (rows // 33 + 7)
    off = torch.cat([starts[:32], torch.tensor([rows], device="cuda")])
    seq = torch.empty(rows, dtype=torch.int32, device="cuda")
    dmt.dmt_sequence_rows(off, seq)
    gate, one = torch.full((rows, cols), 60.0, dtype=torch.bfloat16, device="cuda"), torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    h, final = torch.empty_like(one), torch.full((32, cols), 7.0, device="cuda")
    ws = torch.empty(dmt.dmt_gated_scan_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    dmt.dmt_gated_scan_fwd(gate, one, h, ws, form="free", sequence_of=seq, sequences=32, final=final)
    count = torch.diff(off).float()
    assert torch.equal(final, count[:, None].expand(-1, cols)) and float(count.max()) < 2 ** 24
    for b in (0, 13, 31):                                   # up to 256 bfloat16 holds every number
        a = int(off[b])
        assert torch.equal(h[a:a + 256, 0].float(), torch.arange(1, 257, device="cuda").float())
