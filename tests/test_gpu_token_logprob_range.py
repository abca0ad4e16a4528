"""Log probabilities over the whole range of finite scores, against float64: finite masks of any size, rows far from zero, rows
whose maximum climbs through the powers of two.

Tolerances, before any run.  u = 2^-24; a row's sums are SUM = 1050 u deep (1024 steps in one lane, then lanes, waves and blocks).
The exponent (x_j - max) log2 e takes a handful of roundings relative to itself: a score at distance d is off by 8 u (2 + d), and the
logarithm of the sum by the terms' errors weighted with their probabilities, 8 u sum p_j d_j, at most 8 u H (H the entropy).
"""
import math

import numpy as np
import pytest
import torch

from oracle import sequence as sq

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -24, "bf16": 1e-37}
U32 = 2.0 ** -24
SUM = 1050 * U32


@pytest.fixture(scope="module")
def dmt():
    import paper_2403_00877_amd as d
    return d


def f64(t):
    return t.detach().cpu().double().numpy()


def close(got, ref, tol, what):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    tol = np.broadcast_to(np.where(np.isfinite(ref), tol, 0), got.shape)
    same = (got == ref) | (np.isnan(got) & np.isnan(ref))
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - ref) <= tol))
    if bad.any():
        at = np.unravel_index(int(np.argmax(bad)), bad.shape)
        raise AssertionError("%s: %d of %d off, first at %s: %r, %r expected, tolerance %g"
                             % (what, int(bad.sum()), bad.size, at, got[at], ref[at], tol[at]))


def in_float32(v):
    """What float32 makes of a distance beyond its range."""
    with np.errstate(over="ignore"):
        return np.where(np.isneginf(v.astype(np.float32)), -np.inf, v)


def forward(dmt, x, targets, k):
    rows, vocab = x.shape
    t = torch.from_numpy(targets.astype(np.int32)).cuda()
    new = lambda *s: torch.full(s, 7.0, device="cuda")
    o = dict(logprob=new(rows), entropy=new(rows), stats=new(rows, 2), top_logprobs=new(rows, k) if k else None,
             top_ids=torch.full((rows, k), 77, dtype=torch.int32, device="cuda") if k else None)
    ws = torch.empty(max(256, dmt.dmt_token_logprob_workspace_bytes(rows, vocab, k)), dtype=torch.uint8, device="cuda")
    dmt.dmt_token_logprob_fwd(x, t, workspace=ws, **o)
    return t, o


def check(dmt, x, targets, ks, copies=1):
    """One oracle run of x's rows for every k; `copies` of the rows in a call have to give the same bits."""
    rows, vocab = x.shape
    dt = {v: n for n, v in DT.items()}[x.dtype]
    x64 = f64(x)
    lp, h, ids, lps = sq.token_logprob(x64, targets, max(ks))
    top = x64.max(1)
    with np.errstate(invalid="ignore"):
        lim = lambda dist, v: SUM + 8 * U32 * (2 + (h if dist.ndim == 1 else h[:, None]) + dist) + 4 * U32 * np.abs(v)
        at = x64[np.arange(rows), targets]
        scores = np.where(ids >= 0, np.take_along_axis(x64, np.maximum(ids, 0), 1), -np.inf)
        lp_tol, lps_tol = lim(top - at, lp), lim(top[:, None] - scores, lps)
    big = x.repeat(copies, 1)
    gl, gh = np.random.default_rng(1).normal(size=(2, rows)).astype(np.float32)
    grads = [(a, b, *sq.token_logprob_bwd(x64, targets, a, b)) for a, b in ((gl, gh), (gl, None), (None, gh))]
    for k in ks:
        t, o = forward(dmt, big, np.tile(targets, copies), k)
        same = lambda v: all(torch.equal(v[:rows].nan_to_num(1.25), v[c * rows:(c + 1) * rows].nan_to_num(1.25)) for c in range(copies))
        assert all(same(v) for v in o.values() if v is not None), "a row's answer depends on where it lies"
        close(o["logprob"][:rows], in_float32(lp), lp_tol, "logprob")
        close(o["entropy"][:rows], h, 2 * SUM * (1 + np.abs(h)) + 8 * U32 * 64, "entropy")
        if k:
            assert (o["top_ids"][:rows].cpu().numpy() == ids[:, :k]).all(), "top items"
            close(o["top_logprobs"][:rows], in_float32(lps[:, :k]), lps_tol[:, :k], "top log probabilities")
        for a, b, ref, size in grads:
            d_a, d_b = (None if g is None else torch.from_numpy(np.tile(g, copies)).cuda() for g in (a, b))
            dx = torch.full_like(big, 7.0)
            dmt.dmt_token_logprob_bwd(big, t, o["stats"], o["entropy"], d_a, d_b, dx)
            assert same(dx)
            with np.errstate(invalid="ignore"):
                p = np.exp(x64 - top[:, None])
                tol = 2 * SUM * (size + (0 if b is None else np.abs(gh)[:, None] * p)) + U[dt] * np.abs(ref) + TINY[dt] + 1e-36
            close(dx[:rows], ref, tol, "dx")


def rows_at(rng, size, vocab, dt):
    """Rows that hold scores of magnitude `size` beside ordinary ones, or only such scores."""
    n = lambda: torch.from_numpy(rng.normal(size=vocab) * 2.5)
    x = [n() for _ in range(12)]
    half = vocab // 2
    x[0][:half] = -size                                               # a mask in front, behind, anywhere, everywhere
    x[1][half:] = -size
    x[2][torch.from_numpy(rng.random(vocab) < 0.5)] = -size
    x[3][:] = -size
    x[4][:] = size
    x[5][0] = size                                                    # one score far above, first, last
    x[6][vocab - 1] = size
    x[7][:half], x[7][half::3] = -size, size                          # both
    x[8][torch.from_numpy(rng.random(vocab) < 0.5)] = -size           # masks of both kinds
    x[8][torch.from_numpy(rng.random(vocab) < 0.3)] = -math.inf
    # neighbours: a few units of the type's last place apart
    ulp = size * 2 * U[dt]
    x[9] = size + torch.from_numpy(rng.integers(-4, 5, vocab) * ulp)
    x[10] = -size + torch.from_numpy(rng.integers(-4, 5, vocab) * ulp)
    x[11] = torch.linspace(-size, size, vocab, dtype=torch.float64)   # every score is a new best one
    return torch.stack(x).to(DT[dt]).cuda()


SIZES = [("f32", s) for s in (1e4, 1e5, 1e6, 3e7, 1e8, 1e9, 5e9, 1e10, 1e12, 1e20, 0.9e30, 1e30, 1.1e30, 1e38)] + \
        [("bf16", s) for s in (1e4, 1e6, 1e9, 1e10, 1e12, 1e20, 1e30, 1e38)] + [("f16", s) for s in (1e3, 1e4, 6e4)]


@pytest.mark.parametrize("vocab", [1, 63, 300, 5003, 70_001])
@pytest.mark.parametrize("dt,size", SIZES)
def test_scores_of_any_size(dmt, dt, size, vocab):
    rng = np.random.default_rng(vocab)
    x = rows_at(rng, size, vocab, dt)
    check(dmt, x, f64(x).argmax(1), (10, 0))
    check(dmt, x, rng.integers(0, vocab, len(x)), (1, 40))


@pytest.mark.parametrize("vocab", [700, 5003])
@pytest.mark.parametrize("dt,size", [s for s in SIZES if s[1] in (1e4, 1e6, 1e9, 1e10, 1e20, 1e30)])
def test_scores_of_any_size_in_many_rows(dmt, dt, size, vocab):
    """As many rows as are taken by a wave each."""
    rng = np.random.default_rng(vocab + 1)
    x = rows_at(rng, size, vocab, dt)
    check(dmt, x, f64(x).argmax(1), (12, 0), copies=350)


@pytest.mark.parametrize("power", range(8, 41, 2))
def test_rows_that_climb_through_a_power_of_two(dmt, power):
    """Scores in rising order on both sides of +-2^power, close enough together for all of them to count: however a sum's terms are
    kept, they have to fit the next ones."""
    rng = np.random.default_rng(power)
    for vocab in (40, 5003, 40_001):
        near = torch.linspace(-6, 6, vocab, dtype=torch.float64)
        x = torch.stack([2.0 ** power + near, -2.0 ** power + near, 2.0 ** power - near, -2.0 ** power - near,
                         torch.where(torch.arange(vocab) % 2 == 0, near, -2.0 ** power + near)]).float().cuda()
        check(dmt, x, f64(x).argmax(1), (5, 0))
        check(dmt, x, rng.integers(0, vocab, len(x)), (5,))
    check(dmt, x[:, :3001].contiguous(), rng.integers(0, 3001, len(x)), (5,), copies=820)


@pytest.mark.parametrize("power", range(8, 41, 4))
def test_gradients_far_from_zero_are_differences(dmt, power):
    """The distribution does not change with a shift of all scores, and neither does its gradient: a row near +-2^power in steps that
    float32 holds there, against the same steps at zero."""
    step = max(2.0 ** (power - 23), 2.0 ** -4) * 4
    rng = np.random.default_rng(power)
    off = rng.integers(0, 60, 2000) * step
    x = torch.from_numpy(np.stack([off, off + 2.0 ** power, off - 2.0 ** (power + 1)])).float().cuda()
    assert (f64(x)[1] - 2.0 ** power == off).all() and (f64(x)[2] + 2.0 ** (power + 1) == off).all()
    t = np.full(3, int(off.argmax()))
    d_t, o = forward(dmt, x, t, 3)
    gl, gh, dx = torch.ones(3, device="cuda"), torch.ones(3, device="cuda"), torch.empty_like(x)
    dmt.dmt_token_logprob_bwd(x, d_t, o["stats"], o["entropy"], gl, gh, dx)
    _, size = sq.token_logprob_bwd(f64(x)[:1], t[:1], np.ones(1), np.ones(1))
    p = np.exp(off - off.max())
    for i in (1, 2):
        assert (o["top_ids"][i] == o["top_ids"][0]).all()
        close(o["logprob"][i], f64(o["logprob"][0]), 2 * (SUM + 8 * U32 * 14), "logprob")
        close(o["entropy"][i], f64(o["entropy"][0]), 2 * (2 * SUM * 9 + 8 * U32 * 64), "entropy")
        close(dx[i], f64(dx[0]), 4 * SUM * (size[0] + p) + 1e-36, "dx")


@pytest.mark.parametrize("vocab", [1, 7, 300, 5003, 70_001])
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_scores_at_the_ends_of_the_type(dmt, dt, vocab):
    """Masks of the lowest value, each answer to the tolerance of its own score's distance."""
    rng = np.random.default_rng(vocab + 2)
    low, high, half = torch.finfo(DT[dt]).min, torch.finfo(DT[dt]).max, vocab // 2
    x = [torch.from_numpy(rng.normal(size=vocab) * 2.5) for _ in range(10)]
    x[0][:half], x[1][half:] = low, low
    x[2][torch.from_numpy(rng.random(vocab) < 0.5)] = low
    x[3][:] = low
    x[4][:], x[4][vocab - 1] = low, 2.0                               # one score left: its log probability is 0
    x[5][:], x[5][0] = low, -3.0
    x[6][:], x[6][half] = -math.inf, low                              # beside masks of -inf, the lowest is a score
    x[7][:] = high
    x[8][:half], x[8][half::2] = low, high
    x[9][half] = high
    x = torch.stack(x).to(DT[dt]).cuda()
    check(dmt, x, f64(x).argmax(1), (10, 0))
    check(dmt, x, rng.integers(0, vocab, len(x)), (3,), copies=1 if vocab > 6000 else 420)
