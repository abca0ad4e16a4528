"""More rows than one launch of 2^32 threads holds: every row is done, positions are the call's own."""
import pytest
import torch

from oracle import sequence as sq

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


# rows that are looked at one by one: on both sides of 2^22, where the blocks of 1024 threads pass a launch, and at the ends
def _picked(rows):
    return [0, 1, (1 << 22) - 2, (1 << 22) - 1, 1 << 22, rows - 2, rows - 1]


def _put(t, at, rows):
    for i, r in zip(at, rows):
        t[i].copy_(r)


def _double(t):
    return t.cpu().double().numpy()


def _rows(t, at):
    return _double(torch.stack([t[i] for i in at]))


def test_layer_norm_fwd_of_more_long_rows_than_a_launch_holds(dmt):
    need(150)
    rows, cols = (1 << 22) + 3, 16_385
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    x.copy_(torch.randn(1, cols, generator=g, device="cuda").expand(rows, cols))
    at = _picked(rows)
    some = torch.randn(len(at), cols, generator=g, device="cuda").to(torch.bfloat16)
    _put(x, at, some)
    same = x[5].clone()
    mean, rstd = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    dmt.dmt_layer_norm_fwd(x, None, None, 1e-5, x, mean, rstd)                  # in place
    y, m, r = sq.layer_norm_fwd(_double(torch.cat([some, same[None]])), None, None, 1e-5)
    deep = 300 * U32                                       # terms of a sum in one lane, then lanes and waves
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert bool((mean[rest] == mean[5]).all()) and bool((rstd[rest] == rstd[5]).all())
    at = at + [5]
    assert (abs(_double(mean[at]) - m) <= deep).all() and (abs(_double(rstd[at]) - r) <= 8 * deep * r).all()
    assert (abs(_rows(x, at) - y) <= UBF * abs(y) + 8 * deep * (2 + abs(y))).all()


def test_layer_norm_bwd_of_more_long_rows_than_a_launch_holds(dmt):
    need(150)
    rows, cols = (1 << 22) + 3, 8193
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    x.copy_(torch.randn(1, cols, generator=g, device="cuda").expand(rows, cols))
    dy = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")           # the other rows have no part in the weights' gradients
    at = _picked(rows)
    some, some_dy = (torch.randn(len(at), cols, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    _put(x, at, some)
    _put(dy, at, some_dy)
    _, m, r = sq.layer_norm_fwd(_double(some), None, None, 1e-5)
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    mean[at], rstd[at] = torch.from_numpy(m).float().cuda(), torch.from_numpy(r).float().cuda()
    dg, db = torch.full((cols,), 7.0, device="cuda"), torch.full((cols,), 7.0, device="cuda")
    ws = torch.empty(dmt.dmt_layer_norm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    dmt.dmt_layer_norm_bwd(x, None, mean, rstd, dy, dy, dg, db, ws)             # in place
    d64 = _double(some_dy)
    rx, rg, rb = sq.layer_norm_bwd(_double(some), None, _double(mean[at]), _double(rstd[at]), d64)
    deep = 300 * U32
    h = abs((_double(some) - m[:, None]) * r[:, None])
    size = 2 * (abs(d64) + 1 + h)
    assert (abs(_rows(dy, at) - rx) <= UBF * abs(rx) + deep * size).all()
    assert (abs(_double(dg) - rg) <= 16 * U32 * (abs(d64) * (h + 4)).sum(0)).all()
    assert (abs(_double(db) - rb) <= 16 * U32 * abs(d64).sum(0)).all()
    _put(dy, at, torch.zeros_like(some_dy))
    for a in range(0, rows, 1 << 20):
        assert not bool(dy[a:a + (1 << 20)].any()), a
