"""More rows than one launch of 2^32 threads holds: every row is done, positions are the call's own."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
UBF = 2.0 ** -8


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


def test_token_logprob_of_more_rows_than_a_launch_holds(dmt):
    """2^26 rows and a few: a wave each in the forward, a block each in the backward."""
    need(24)
    rows, vocab = (1 << 26) + 5, 3
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(rows, vocab, generator=g, device="cuda", dtype=torch.bfloat16)
    t = torch.randint(vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    t[rows - 2] = vocab
    lp, h = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    st, top = torch.full((rows, 2), 7.0, device="cuda"), torch.full((rows, 1), 7, device="cuda", dtype=torch.int32)
    bad = torch.full((1,), -1, dtype=torch.int64, device="cuda")
    ws = torch.empty(max(256, dmt.dmt_token_logprob_workspace_bytes(rows, vocab, 1)), dtype=torch.uint8, device="cuda")
    dmt.dmt_token_logprob_fwd(x, t, lp, h, top, None, st, ws, bad)
    assert int(bad) == rows - 2
    gl = torch.rand(rows, generator=g, device="cuda")
    gl[rows - 2] = 0.0                                    # no target
    dx = torch.full_like(x, 7.0)
    dmt.dmt_token_logprob_bwd(x, t, st, h, gl, None, dx)
    for a in range(0, rows, 1 << 23):                     # (three terms a row: a few roundings)
        b = min(rows, a + (1 << 23))
        x64 = x[a:b].double()
        logp = torch.log_softmax(x64, 1)
        at = t[a:b].long().clamp(max=vocab - 1)[:, None]
        there = t[a:b] < vocab
        ref = torch.where(there, logp.gather(1, at)[:, 0], 0.0)
        assert float((lp[a:b] - ref).abs().max()) <= 64 * U32 * 12, a
        p = logp.exp()
        assert float((h[a:b] + (p * logp).sum(1)).abs().max()) <= 64 * U32 * 12, a
        best = x64.max(1, keepdim=True).values
        assert bool((top[a:b, 0] == (x64 == best).int().argmax(1)).all()), a
        assert bool((st[a:b, 0] == best[:, 0]).all()), a
        want = gl[a:b, None].double() * (torch.zeros_like(p).scatter_(1, at, 1.0) - p)
        assert bool(((dx[a:b] - want).abs() <= UBF * want.abs() + 64 * U32).all()), a


def test_embed_fwd_of_more_ids_than_a_launch_holds(dmt):
    """2^26 ids and a few, a wave each."""
    need(40)
    n, rows, cols = (1 << 26) + 3, 1000, 129
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    table = torch.randn(rows, cols, generator=g, device="cuda")
    ids = torch.randint(-1, rows, (n,), generator=g, device="cuda", dtype=torch.int32)
    ids[n - 2] = rows
    out = torch.full((n, cols), 7.0, dtype=torch.float16, device="cuda")
    bad = torch.full((1,), -1, dtype=torch.int64, device="cuda")
    dmt.dmt_embed_fwd(table, ids, out, first_bad=bad)
    assert int(bad) == n - 2
    there = torch.cat([table, torch.zeros(1, cols, device="cuda")]).half()      # row `rows`: of absent ids
    for a in range(0, n, 1 << 24):
        i = ids[a:a + (1 << 24)].long()
        assert torch.equal(out[a:a + (1 << 24)], there[torch.where(i < 0, rows, i)]), a
