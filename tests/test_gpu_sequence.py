"""The sequence branch's kernels against float64, through the binding.

Tolerances come from the number format and the depth of the sums, before any run:
  u16 (2^-8 bf16, 2^-11 f16) and u32 = 2^-24 are the largest relative errors of one rounding;
  a sum of n terms is off by at most (its depth) * u32 * (sum of the terms' magnitudes), the depth being n
  for one running sum and far less for a sum over lanes, waves and blocks.
"""
import math

import numpy as np
import pytest
import torch

from oracle import sequence as sq

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -24, "bf16": 1e-37}      # where a type runs out of small values
U32 = 2.0 ** -24


@pytest.fixture(scope="module")
def dmt():
    import paper_2403_00877_amd as d
    return d


def f64(t):
    return t.detach().cpu().double().numpy()


def matrix(rng, rows, cols, dtype, pad=0, shift=0, scale=1.0, mean=0.0):
    """A seeded [rows][cols] matrix of row stride cols + pad that starts `shift` elements into its
    memory, NaN all around it."""
    buf = torch.full((shift + rows * (cols + pad) + 64,), float("nan"), dtype=DT[dtype], device="cuda")
    m = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if rows:
        m.copy_(torch.from_numpy(rng.normal(size=(rows, cols)) * scale + mean))
    return m


def blank(rows, cols, dtype, pad=0, shift=0):
    """An output like `matrix`, and the memory around it to be checked by `untouched`."""
    buf = torch.full((shift + rows * (cols + pad) + 64,), 7.0, dtype=DT[dtype], device="cuda")
    return buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols], (buf, rows, cols, pad, shift)


def untouched(around):
    buf, rows, cols, pad, shift = around
    b = buf.clone()
    b[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = 7.0
    assert bool((b == 7.0).all()), "written outside the matrix"


def close(got, ref, tol, what):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    ref, tol = np.broadcast_to(ref, got.shape), np.broadcast_to(tol, got.shape)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    same = (got == ref) | (np.isnan(got) & np.isnan(ref))
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - ref) <= tol))
    if bad.any():
        at = np.unravel_index(int(np.argmax(bad)), bad.shape)
        raise AssertionError("%s: %d of %d off, first at %s: %r, %r expected, tolerance %g"
                             % (what, int(bad.sum()), bad.size, at, got[at], ref[at], tol[at]))


def bytes_buf(n):
    return torch.empty(max(256, n), dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------ embedding

SHAPES = [(1, 1, 1, 0, 0), (1, 50, 128, 0, 0), (7, 3, 5, 1, 1), (64, 10, 8, 0, 0), (333, 1000, 33, 3, 1),
          (1000, 77, 100, 4, 2), (2049, 5000, 64, 0, 0), (500, 40, 1030, 2, 3), (129, 20, 513, 0, 0), (40, 9, 4099, 1, 1)]


def some_ids(rng, n, rows, kind):
    if kind == "skew":
        ids = np.minimum(rows - 1, (rows * rng.random(n) ** 4).astype(np.int64))
    elif kind == "one":
        ids = np.full(n, rows // 2)
    elif kind == "sorted":
        ids = np.sort(rng.integers(0, rows, n))
    else:
        ids = rng.integers(0, rows, n)
    ids = ids.astype(np.int32)
    if kind == "holes":
        ids[rng.random(n) < 0.3] = -1
        ids[rng.random(n) < 0.1] = rows
        ids[rng.random(n) < 0.05] = np.iinfo(np.int32).max
        ids[rng.random(n) < 0.05] = np.iinfo(np.int32).min
    if kind == "none":
        ids[:] = -3
    return ids


@pytest.mark.parametrize("td,od", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f16", "bf16"), ("bf16", "f32"),
                                   ("f32", "f16")])
@pytest.mark.parametrize("n,rows,cols,pad,shift", SHAPES)
def test_embed_fwd(dmt, n, rows, cols, pad, shift, td, od):
    rng = np.random.default_rng(n + cols)
    table = matrix(rng, rows, cols, td, pad, shift)
    scale = float(np.float32(math.sqrt(cols)))
    for kind in ("uniform", "holes"):
        ids = some_ids(rng, n, rows, kind)
        out, around = blank(n, cols, od, pad, shift)
        bad = torch.full((1,), -1, dtype=torch.int64, device="cuda")
        dmt.dmt_embed_fwd(table, torch.from_numpy(ids).cuda(), out, scale, bad)
        ref = sq.embed_fwd(f64(table), ids, scale)
        close(out, ref, (U[od] + 2 * U32) * np.abs(ref) + TINY[od], "rows")      # the product, then the type
        untouched(around)
        over = np.nonzero(ids >= rows)[0]
        assert int(bad.cpu()) == (over[0] if len(over) else -1)


@pytest.mark.parametrize("kind", ["uniform", "skew", "one", "sorted", "holes", "none"])
@pytest.mark.parametrize("gd", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,rows,cols,pad,shift", SHAPES + [(0, 5, 7, 0, 0), (4096, 300, 24, 0, 0), (4097, 300, 24, 0, 0),
                                                          (9000, 3000, 16, 1, 0), (4500, 3, 5, 1, 1),
                                                          (4200, 40, 1030, 2, 3), (5000, 333, 130, 0, 0), (66_000, 70, 40, 3, 1)])
def test_embed_bwd(dmt, n, rows, cols, pad, shift, gd, kind):
    rng = np.random.default_rng(n + 3 * cols)
    ids = some_ids(rng, n, rows, kind)
    d_ids = torch.from_numpy(ids).cuda()
    grad = matrix(rng, n, cols, gd, pad, shift)
    scale = 0.75
    ref, size = sq.embed_bwd(ids, f64(grad), rows, scale)
    count = np.bincount(ids[(ids >= 0) & (ids < rows)], minlength=rows)[:, None]
    tol = (count + 2) * U32 * size
    ws = bytes_buf(dmt.dmt_embed_bwd_workspace_bytes(n, rows, cols))
    ws.fill_(0xA5)                                       # scratch starts as anything
    out, around = blank(rows, cols, "f32", pad, shift)
    bad = torch.full((1,), -1, dtype=torch.int64, device="cuda")
    dmt.dmt_embed_bwd(d_ids, grad, out, ws, scale, first_bad=bad)
    close(out, ref, tol, "gradient")
    untouched(around)
    over = np.nonzero(ids >= rows)[0]
    assert int(bad.cpu()) == (over[0] if len(over) else -1)
    again, _ = blank(rows, cols, "f32", pad, shift)
    dmt.dmt_embed_bwd(d_ids, grad, again, ws, scale)
    assert torch.equal(out, again), "another run, other bits"
    # added to what is there; rows without an id keep their bits
    acc = matrix(rng, rows, cols, "f32", pad, shift)
    before = f64(acc)
    dmt.dmt_embed_bwd(d_ids, grad, acc, ws, scale, accumulate=True)
    close(acc, before + ref, tol + 2 * U32 * (np.abs(before) + size), "accumulated")
    assert (f64(acc)[count[:, 0] == 0] == before[count[:, 0] == 0]).all()


@pytest.mark.parametrize("n,rows,cols,kind", [(70_000, 20_000, 32, "skew"), (70_000, 1_500_000, 8, "uniform"),
                                              (150_000, 2_000, 16, "one"), (300_000, 100_000, 16, "skew"),
                                              (200_000, 3_000_000, 4, "holes"), (1_200_000, 5_000, 8, "skew"),
                                              (20_000, 700_000, 12, "skew"), (40_000, 2_500_000, 4, "uniform")])
def test_embed_bwd_of_many(dmt, n, rows, cols, kind):
    """Sizes past every line between the ways to sort, small integers for gradients: every sum is exact."""
    rng = np.random.default_rng(n)
    ids = some_ids(rng, n, rows, kind)
    g = rng.integers(-8, 9, size=(n, cols))
    ref = np.zeros((rows, cols), np.int64)
    ok = (ids >= 0) & (ids < rows)
    np.add.at(ref, ids[ok], g[ok])
    ws = bytes_buf(dmt.dmt_embed_bwd_workspace_bytes(n, rows, cols))
    for gd in ("f32", "bf16"):
        out, around = blank(rows, cols, "f32")
        dmt.dmt_embed_bwd(torch.from_numpy(ids).cuda(), torch.from_numpy(g).cuda().to(DT[gd]), out, ws)
        assert bool((out == torch.from_numpy(ref).cuda()).all())
        untouched(around)


def test_embed_past_32_bit_offsets(dmt):
    """A table of more than 2^32 elements: its last rows, forward and (accumulating) backward."""
    rows, cols = 34_000_001, 128
    table = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([rows - 1, 0, rows - 2, rows - 1], dtype=torch.int32, device="cuda")
    some = torch.randn(3, cols, device="cuda").to(torch.bfloat16)
    table[[rows - 1, 0, rows - 2]] = some
    out = torch.empty(4, cols, dtype=torch.bfloat16, device="cuda")
    dmt.dmt_embed_fwd(table, ids, out)
    assert torch.equal(out, some[[0, 1, 2, 0]])
    del table
    grad_table = torch.empty(rows, cols, dtype=torch.float32, device="cuda")
    grad_table[[rows - 1, 0, rows - 2, 5]] = 1.0
    ws = bytes_buf(dmt.dmt_embed_bwd_workspace_bytes(4, rows, cols))
    dmt.dmt_embed_bwd(ids, out, grad_table, ws, accumulate=True)
    s = some.float()
    assert torch.equal(grad_table[[rows - 1, 0, rows - 2, 5]],
                       torch.stack([1 + (s[0] + s[0]), 1 + s[1], 1 + s[2], torch.ones_like(s[0])]))


# ------------------------------------------------------------------ layer norm

NORM = [(1, 1), (3, 2), (5, 7), (17, 8), (9, 64), (33, 65), (64, 100), (200, 128), (70, 129), (37, 255), (41, 256),
        (13, 511), (19, 512), (29, 1000), (31, 1024), (23, 1052), (11, 2048), (7, 2049), (9, 4095), (6, 4096),
        (5, 6001), (4, 8192), (3, 16_384), (2, 33_000), (2, 70_001), (1, 131_072), (700, 48), (1500, 256), (0, 16)]


def norm_case(rng, rows, cols, dt, wd, pad, shift):
    x = matrix(rng, rows, cols, dt, pad, shift, scale=1.5, mean=0.5)
    gamma = matrix(rng, 1, cols, wd, 0, shift, scale=0.5, mean=1.0)[0]
    beta = matrix(rng, 1, cols, wd, 0, shift)[0]
    return x, gamma, beta


# Sums over a row run over at most 256 terms in one lane (then over lanes and waves): depth 280.  The mean is off by
# 280 u32 mean|x|, at most 280 u32 * 2 std here, and 1/std by as much relatively, so h = (x - mean)/std by
# 280 u32 (2 + |h|) and a few roundings.
DEEP = 300 * U32


@pytest.mark.parametrize("dt,wd", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f16", "f32")])
@pytest.mark.parametrize("rows,cols", NORM)
def test_layer_norm_fwd(dmt, rows, cols, dt, wd):
    rng = np.random.default_rng(rows * 7 + cols)
    for pad, shift in ((0, 0), (3, 1)):
        x, gamma, beta = norm_case(rng, rows, cols, dt, wd, pad, shift)
        y, around = blank(rows, cols, dt, pad, shift)
        mean, rstd = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
        dmt.dmt_layer_norm_fwd(x, gamma, beta, 1e-5, y, mean, rstd)
        g, b = f64(gamma), f64(beta)
        ry, rm, rr = sq.layer_norm_fwd(f64(x), g, b, 1e-5)
        close(mean, rm, DEEP * np.abs(f64(x)).mean(1) if rows else 0, "mean")
        spread = 1 + (np.abs(f64(x)).mean(1) if rows else 0) * rr      # mean's error in units of std (small rows: std may be small)
        close(rstd, rr, 4 * DEEP * rr * spread ** 2, "rstd")
        h = np.abs((f64(x) - rm[:, None]) * rr[:, None])
        close(y, ry, U[dt] * np.abs(ry) + TINY[dt] + 4 * DEEP * (spread[:, None] ** 2 if rows else 1) * (np.abs(g) * (2 + h)) + 4 * U32 * np.abs(b), "y")
        untouched(around)
        # without weights, and in place
        plain, _ = blank(rows, cols, dt, pad, shift)
        dmt.dmt_layer_norm_fwd(x, None, None, 1e-5, plain)
        ones = torch.empty(rows, cols, dtype=DT[dt], device="cuda")
        dmt.dmt_layer_norm_fwd(x, torch.ones_like(gamma), torch.zeros_like(beta), 1e-5, ones)
        assert torch.equal(plain.contiguous(), ones)
        dmt.dmt_layer_norm_fwd(x, gamma, beta, 1e-5, x)
        assert torch.equal(x, y)


def test_layer_norm_fwd_of_a_constant_row_and_of_rows_that_are_not_finite(dmt):
    x = torch.full((4, 100), 3.0, device="cuda")
    x[1, 5] = float("nan")
    x[2, 99] = float("inf")
    y = torch.empty_like(x)
    dmt.dmt_layer_norm_fwd(x, None, None, 1e-5, y)
    assert bool((y[[0, 3]] == 0).all()) and bool(y[1].isnan().all()) and bool(y[2].isnan().all())


@pytest.mark.parametrize("dt,gd,wd", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "bf16"),
                                      ("f16", "f16", "f32"), ("f16", "f32", "f16")])
@pytest.mark.parametrize("rows,cols", NORM)
def test_layer_norm_bwd(dmt, rows, cols, dt, gd, wd):
    rng = np.random.default_rng(rows * 5 + cols)
    for pad, shift in ((0, 0), (3, 1)):
        x, gamma, _ = norm_case(rng, rows, cols, dt, wd, pad, shift)
        dy = matrix(rng, rows, cols, gd, pad, shift)
        _, m, r = sq.layer_norm_fwd(f64(x), None, None, 1e-5)
        mean, rstd = torch.from_numpy(m).float().cuda(), torch.from_numpy(r).float().cuda()
        dx, around = blank(rows, cols, gd, pad, shift)
        dg, db = torch.full((cols,), 7.0, device="cuda"), torch.full((cols,), 7.0, device="cuda")
        ws = bytes_buf(dmt.dmt_layer_norm_bwd_workspace_bytes(rows, cols))
        ws.fill_(0xA5)
        dmt.dmt_layer_norm_bwd(x, gamma, mean, rstd, dy, dx, dg, db, ws)
        g64, x64, dy64, m64, r64 = f64(gamma), f64(x), f64(dy), f64(mean)[:, None], f64(rstd)[:, None]
        rx, rg, rb = sq.layer_norm_bwd(x64, g64, m64[:, 0], r64[:, 0], dy64)
        h = np.abs((x64 - m64) * r64)
        h_err = 4 * U32 * (np.abs(x64) + np.abs(m64)) * r64              # of (x - mean) * rstd
        g = np.abs(dy64 * g64)
        if rows:
            size = r64 * (g + g.mean(1, keepdims=True) + h * (g * h).mean(1, keepdims=True))
            slack = r64 * (h_err * (g * h).mean(1, keepdims=True) + h * (g * h_err).mean(1, keepdims=True))
            close(dx, rx, U[gd] * np.abs(rx) + TINY[gd] + DEEP * size + slack, "dx")
        untouched(around)
        deep = (rows + 8) * U32
        close(dg, rg, deep * (np.abs(dy64) * h).sum(0) + (np.abs(dy64) * h_err).sum(0), "dgamma")
        close(db, rb, deep * np.abs(dy64).sum(0), "dbeta")
        # the weights' gradients repeat bit for bit; dx alone; one of the two; in place
        dg2, db2 = torch.empty_like(dg), torch.empty_like(db)
        dmt.dmt_layer_norm_bwd(x, gamma, mean, rstd, dy, dx, dg2, None, ws)
        dmt.dmt_layer_norm_bwd(x, gamma, mean, rstd, dy, dx, None, db2, ws)
        assert torch.equal(dg, dg2) and torch.equal(db, db2)
        alone, _ = blank(rows, cols, gd, pad, shift)
        dmt.dmt_layer_norm_bwd(x, gamma, mean, rstd, dy, alone)
        assert torch.equal(dx, alone)
        dmt.dmt_layer_norm_bwd(x, gamma, mean, rstd, dy, dy, dg2, db2, ws)
        assert torch.equal(dx, dy) and torch.equal(dg, dg2) and torch.equal(db, db2)


MANY = [(513, 5), (5000, 17), (900, 33), (2100, 60), (800, 127), (2000, 130), (600, 200), (520, 511), (600, 1052), (513, 2049), (514, 4100),
        (700, 8192), (520, 9001)]


@pytest.mark.parametrize("dt,gd,wd", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f16", "f32", "f16")])
@pytest.mark.parametrize("rows,cols", MANY)
def test_layer_norm_of_many_rows(dmt, rows, cols, dt, gd, wd):
    """More rows than one launch of the backward takes, at every number of lanes a row."""
    test_layer_norm_fwd(dmt, rows, cols, dt, wd)
    test_layer_norm_bwd(dmt, rows, cols, dt, gd, wd)


def test_layer_norm_gradients_against_differences(dmt):
    """Directional differences of the forward, computed in float64, against the kernel's gradients."""
    rng = np.random.default_rng(3)
    for rows, cols in ((3, 5), (40, 130), (4, 3001)):
        x, gamma, beta = norm_case(rng, rows, cols, "f32", "f32", 0, 0)
        dy = matrix(rng, rows, cols, "f32")
        y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        dmt.dmt_layer_norm_fwd(x, gamma, beta, 1e-5, y, mean, rstd)
        dx, dg, db = torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        dmt.dmt_layer_norm_bwd(x, gamma, mean, rstd, dy, dx, dg, db,
                               bytes_buf(dmt.dmt_layer_norm_bwd_workspace_bytes(rows, cols)))
        args, grads, d = [f64(x), f64(gamma), f64(beta)], [f64(dx), f64(dg), f64(db)], f64(dy)
        loss = lambda a: float((sq.layer_norm_fwd(*a, 1e-5)[0] * d).sum())
        for i in range(3):
            for _ in range(4):
                v = rng.normal(size=args[i].shape)
                e = 1e-6
                up, down = list(args), list(args)
                up[i], down[i] = args[i] + e * v, args[i] - e * v
                diff, size = (loss(up) - loss(down)) / (2 * e), np.abs(grads[i] * v).sum()
                assert abs(diff - (grads[i] * v).sum()) <= 1e-4 * size, (rows, cols, i)


# ------------------------------------------------------------------ log probabilities

# A row's sums take at most 1024 steps in one lane at these sizes, then lanes, waves and blocks: depth 1050.
SUM = 1050 * U32


def check_logprob(dmt, x, targets, k, gl=None, gh=None, with_bad=False):
    rows, vocab = x.shape
    dt = {v: n for n, v in DT.items()}[x.dtype]
    t = torch.from_numpy(targets.astype(np.int32)).cuda()
    x64 = f64(x)
    lp, h, ids, lps = sq.token_logprob(x64, targets, k)
    new = lambda *s: torch.full(s, 7.0, device="cuda")
    logprob, entropy, stats, top_lp = new(rows), new(rows), new(rows, 2), new(rows, k)
    top = torch.full((rows, k), 77, dtype=torch.int32, device="cuda")
    ws = bytes_buf(dmt.dmt_token_logprob_workspace_bytes(rows, vocab, k))
    ws.fill_(0xA5)
    bad = torch.full((1,), -1, dtype=torch.int64, device="cuda")
    dmt.dmt_token_logprob_fwd(x, t, logprob, entropy, top if k else None, top_lp if k else None, stats, ws, bad)
    with np.errstate(invalid="ignore", over="ignore"):
        # x - max and its exponential round relative to |x - max|; the logarithm of the sum is off by the sum's depth
        # (a distance beyond float32's range is -inf)
        far = np.where(np.isfinite(x64), np.abs(x64), 0).max(1)
        tol = SUM + 8 * U32 * (2 + far)
        over = lambda v: np.where(np.isneginf(v.astype(np.float32)), -np.inf, v)
        close(logprob, over(lp), np.where(np.isfinite(lp), tol + 4 * U32 * np.abs(lp), 0), "logprob")
        close(entropy, h, 2 * SUM * (1 + np.abs(h)) + 8 * U32 * 64, "entropy")
        clean = ~np.isnan(x64).any(1) & ~np.isposinf(x64).any(1)
        if k:
            assert (top.cpu().numpy()[clean] == ids[clean]).all(), "top items"
            close(f64(top_lp)[clean], over(lps)[clean], (tol[:, None] + 4 * U32 * np.abs(lps))[clean], "top log probabilities")
            assert ((top.cpu().numpy() >= -1) & (top.cpu().numpy() < vocab)).all()
    over_t = np.nonzero(targets >= vocab)[0]
    assert int(bad.cpu()) == (over_t[0] if len(over_t) else -1)
    if gl is None:
        return
    d_gl, d_gh = torch.from_numpy(gl).float().cuda(), torch.from_numpy(gh).float().cuda()
    for a, b in ((d_gl, d_gh), (d_gl, None), (None, d_gh)):
        ref, size = sq.token_logprob_bwd(x64, targets, None if a is None else f64(a), None if b is None else f64(b))
        dx, around = blank(rows, vocab, dt, x.stride(0) - vocab if rows > 1 else 0)
        dmt.dmt_token_logprob_bwd(x, t, stats, entropy, a, b, dx)
        with np.errstate(invalid="ignore"):
            lim = 2 * SUM * (size + (0 if b is None else np.abs(f64(b))[:, None] * np.exp(np.minimum(0, x64 - x64.max(1, keepdims=True))))) + U[dt] * np.abs(ref) + TINY[dt] + 1e-36
            close(dx, ref, np.where(np.isfinite(lim), lim, 0), "dx")
        untouched(around)
        if a is not None and b is not None:
            mine = x.clone()
            dmt.dmt_token_logprob_bwd(mine, t, stats, entropy, a, b, mine)
            assert torch.equal(mine, dx) or bool(dx.isnan().any())


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab,k", [
    (1, 1, 1), (3, 2, 2), (2, 5, 8), (5, 63, 1), (4, 64, 5), (7, 65, 10), (3, 255, 3), (6, 256, 20), (5, 257, 64),
    (3, 1000, 0), (9, 1001, 33), (2, 4095, 10), (2, 4096, 50), (3, 4097, 10), (2, 8191, 7), (4, 8193, 10), (2, 12_289, 64),
    (3, 16_384, 10), (2, 16_385, 20), (1, 20_011, 64), (3, 65_536, 10), (1, 100_003, 50), (1, 262_144, 10), (0, 10, 3)])
def test_token_logprob(dmt, rows, vocab, k, dt):
    rng = np.random.default_rng(vocab + rows)
    for pad, shift in ((0, 0), (3, 1)):
        x = matrix(rng, rows, vocab, dt, pad, shift, scale=2.5)
        t = rng.integers(0, vocab, rows)
        if rows > 2:
            t[1], t[2] = -1, vocab + 5
        check_logprob(dmt, x, t, k, rng.normal(size=rows), rng.normal(size=rows))


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [7, 300, 5000, 20_000, 70_001])
def test_token_logprob_of_awkward_rows(dmt, vocab, dt):
    """Ties, sorted rows, masks of -inf and of the lowest value, rows that hold nothing, one item far above."""
    rng = np.random.default_rng(vocab)
    low = float(torch.finfo(DT[dt]).min)
    x = torch.empty(16, vocab, dtype=torch.float64)
    x[0] = 0.0                                                        # all alike
    x[1] = torch.arange(vocab, dtype=torch.float64) * (20.0 / vocab)  # ascending: every score is a new best one
    x[2] = -x[1]
    x[3] = torch.from_numpy(rng.integers(0, 4, vocab) * 1.0)          # four values
    x[4] = torch.from_numpy(rng.normal(size=vocab))
    x[4][torch.from_numpy(rng.random(vocab) < 0.7)] = -math.inf
    x[5] = -math.inf                                                  # nothing left
    x[6] = -math.inf
    x[6, vocab // 2] = 1.5                                            # one item left
    x[7] = low                                                        # all at the lowest value
    x[8] = low
    x[8, vocab - 1] = 2.0
    x[9] = torch.from_numpy(rng.normal(size=vocab))
    x[9, 1] = 60.0                                                    # certain
    x[10] = -math.inf
    x[10, ::3] = torch.from_numpy(rng.normal(size=len(range(0, vocab, 3))))
    x[11] = torch.where(torch.arange(vocab) % 2 == 0, 0.0, -0.0)      # zeros of both signs tie
    x[12] = torch.from_numpy(rng.normal(size=vocab) * 1e-3 - 1000.0)
    x[13] = -math.inf
    x[13, -min(vocab, 3):] = torch.tensor([0.5, 1.0, 0.5])[:min(vocab, 3)]
    x[14] = torch.where(torch.arange(vocab) < vocab - 5, -5.0, 5.0)   # the best lie at the end, alike
    x[15] = torch.from_numpy(np.repeat(rng.normal(size=vocab // 64 + 1), 64)[:vocab])   # a lane's neighbours alike
    x = x.to(DT[dt]).cuda()
    t = rng.integers(0, vocab, 16)
    t[6], t[8], t[5], t[9] = vocab // 2, vocab - 1, 0, 2
    for k in (1, 5, 10, 64):
        check_logprob(dmt, x, t, k, rng.normal(size=16), rng.normal(size=16))
    t[5] = t[4] = -1
    check_logprob(dmt, x, t, 3, rng.normal(size=16), rng.normal(size=16))


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("copies,vocab", [(90, 9001), (150, 33_003), (47, 70_001)])
def test_token_logprob_of_many_awkward_rows(dmt, copies, vocab, dt):
    """As many rows as let a block walk through several thousand scores of one: ties, sorted rows, scores that all hide in one
    wave's part, few scores that are left, the best ones in front or at the end."""
    rng = np.random.default_rng(vocab + copies)
    low = float(torch.finfo(DT[dt]).min)
    at = np.arange(vocab)
    x = np.full((12, vocab), -np.inf)
    x[0] = 1.0
    x[1] = at * (20.0 / vocab)
    x[2] = -x[1]
    x[3] = rng.integers(0, 4, vocab)
    x[4] = np.where(at // 512 % 4 == 1, rng.normal(size=vocab), -9.0)
    x[5, rng.choice(vocab, 30, False)] = rng.normal(size=30)
    x[6] = low
    x[6, ::97] = rng.normal(size=len(x[6, ::97]))
    x[7] = np.where(at % 2 == 0, 0.0, -0.0)
    x[7, vocab - 9:] = 3.0
    x[8] = np.where(at < 40, 7.0, rng.normal(size=vocab))
    x[9] = np.where(at % 64 == 5, rng.normal(size=vocab) + 4, rng.normal(size=vocab))
    x[10] = rng.normal(size=vocab)
    x = torch.from_numpy(x).to(DT[dt])
    big = x.cuda().repeat(copies, 1)
    rows = big.shape[0]
    t = rng.integers(0, vocab, 12)
    td = torch.from_numpy(np.tile(t, copies).astype(np.int32)).cuda()
    x64 = f64(x)
    far = np.where(np.isfinite(x64), np.abs(x64), 0).max(1)
    tol = SUM + 8 * U32 * (2 + far)
    over = lambda v: np.where(np.isneginf(v.astype(np.float32)), -np.inf, v)
    for k in (1, 7, 20, 64):
        with np.errstate(invalid="ignore", over="ignore"):
            lp, h, ids, lps = sq.token_logprob(x64, t, k)
        logprob, entropy, top_lp = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, k, device="cuda")
        top = torch.full((rows, k), 77, dtype=torch.int32, device="cuda")
        ws = bytes_buf(dmt.dmt_token_logprob_workspace_bytes(rows, vocab, k))
        dmt.dmt_token_logprob_fwd(big, td, logprob, entropy, top, top_lp, None, ws)
        with np.errstate(invalid="ignore", over="ignore"):
            for c in range(copies):
                mine = slice(12 * c, 12 * c + 12)
                assert (top[mine].cpu().numpy() == ids).all(), (c, k)
                close(logprob[mine], over(lp), np.where(np.isfinite(lp), tol + 4 * U32 * np.abs(lp), 0), "logprob")
                close(entropy[mine], h, 2 * SUM * (1 + np.abs(h)) + 8 * U32 * 64, "entropy")
                close(f64(top_lp[mine]), over(lps), tol[:, None] + 4 * U32 * np.abs(lps), "top log probabilities")


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("copies,vocab", [(175, 700), (171, 2049), (342, 1000), (343, 5003), (350, 17_001)])
def test_token_logprob_of_very_many_awkward_rows(dmt, copies, vocab, dt):
    """As many rows as are taken by a wave each."""
    test_token_logprob_of_many_awkward_rows(dmt, copies, vocab, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(4099, 64), (4099, 3001), (5, 511), (4097, 8190)])
def test_token_logprob_of_very_many_rows_without_lists(dmt, rows, vocab, dt):
    rng = np.random.default_rng(vocab + rows)
    x = matrix(rng, rows, vocab, dt, 3, 1, scale=2.5)
    t = rng.integers(0, vocab, rows)
    t[rows // 2], t[rows - 1] = -1, vocab + 5
    check_logprob(dmt, x, t, 0)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [5, 300, 20_000])
def test_token_logprob_of_rows_that_are_not_finite(dmt, vocab, dt):
    rng = np.random.default_rng(vocab)
    x = rng.normal(size=(4, vocab))
    x[0, vocab // 3], x[1, vocab - 1], x[2, 0] = np.nan, np.inf, np.nan
    x[2, 1:] = -np.inf
    x = torch.from_numpy(x).to(DT[dt]).cuda()
    check_logprob(dmt, x, np.array([0, 0, 0, 0]), 4)


def test_token_logprob_past_32_bit_offsets(dmt):
    """Rows that lie more than 2^32 elements apart."""
    vocab = 1000
    buf = torch.empty((1 << 32) + vocab + 8, dtype=torch.float16, device="cuda")
    x = torch.as_strided(buf, (2, vocab), ((1 << 32) + 3, 1))
    x.copy_(torch.randn(2, vocab, device="cuda"))
    t = torch.tensor([3, 999], dtype=torch.int32, device="cuda")
    lp, h, st = torch.empty(2, device="cuda"), torch.empty(2, device="cuda"), torch.empty(2, 2, device="cuda")
    dmt.dmt_token_logprob_fwd(x, t, lp, h, stats=st, workspace=bytes_buf(dmt.dmt_token_logprob_workspace_bytes(2, vocab, 0)))
    ref = sq.token_logprob(f64(x), t.cpu().numpy(), 0)
    close(lp, ref[0], SUM + 1e-5, "logprob")
    gl = torch.ones(2, device="cuda")
    rx, size = sq.token_logprob_bwd(f64(x), t.cpu().numpy(), np.ones(2), None)
    dmt.dmt_token_logprob_bwd(x, t, st, None, gl, None, x)
    close(x, rx, 2 * SUM * size + U["f16"] * np.abs(rx) + TINY["f16"], "dx in place")


def test_token_logprob_gradient_against_differences(dmt):
    rng = np.random.default_rng(8)
    x = matrix(rng, 6, 700, "f32", scale=2.0)
    t = rng.integers(0, 700, 6)
    gl, gh = rng.normal(size=6).astype(np.float32), rng.normal(size=6).astype(np.float32)
    d_t = torch.from_numpy(t.astype(np.int32)).cuda()
    h, st, dx = torch.empty(6, device="cuda"), torch.empty(6, 2, device="cuda"), torch.empty_like(x)
    dmt.dmt_token_logprob_fwd(x, d_t, None, h, stats=st, workspace=bytes_buf(dmt.dmt_token_logprob_workspace_bytes(6, 700, 0)))
    dmt.dmt_token_logprob_bwd(x, d_t, st, h, torch.from_numpy(gl).cuda(), torch.from_numpy(gh).cuda(), dx)

    def loss(v):
        lp, e, _, _ = sq.token_logprob(v, t, 0)
        return float((lp * gl + e * gh).sum())

    x64 = f64(x)
    for _ in range(6):
        v = rng.normal(size=x64.shape)
        diff = (loss(x64 + 1e-6 * v) - loss(x64 - 1e-6 * v)) / 2e-6
        assert abs(diff - (f64(dx) * v).sum()) <= 1e-4 * np.abs(f64(dx) * v).sum()


# ------------------------------------------------------------------ norm and clipping


def grads_of(rng, sizes, kinds, shift=0, scale=1.0):
    out = []
    for n, kind in zip(sizes, kinds):
        buf = torch.full((n + shift + 8,), float("nan"), dtype=DT[kind], device="cuda")
        buf[shift:shift + n] = torch.from_numpy(rng.normal(size=n) * scale)
        out.append(buf[shift:shift + n])
    return out


def check_clip(dmt, grads, max_norm):
    names = {v: n for n, v in DT.items()}
    host = [f64(g) for g in grads]
    norm, coef = sq.grad_clip(host, max_norm)
    lst = dmt.make_grad_list(grads)
    ws = bytes_buf(dmt.dmt_grad_norm_workspace_bytes(lst))
    ws.fill_(0xA5)
    got = torch.full((1,), 7.0, device="cuda")
    dmt.dmt_grad_norm(lst, got, ws)
    # squares and sums in float64, then one rounding
    norm32 = math.inf if norm > 3.4028235e38 else norm
    close(got, np.array([norm32]), 2 * U32 * norm if math.isfinite(norm32) else 0, "norm")
    outs = [torch.full((g.numel() + 8,), 7.0, dtype=g.dtype, device="cuda") for g in grads]
    views = [o[3:3 + g.numel()] for o, g in zip(outs, grads)]
    got.fill_(7.0)
    dmt.dmt_grad_clip(dmt.make_grad_list(grads, views), max_norm, got, ws)
    close(got, np.array([norm32]), 2 * U32 * norm if math.isfinite(norm32) else 0, "norm of the clipping")
    if norm32 == math.inf:
        coef = 0.0
    for o, v, h in zip(outs, views, host):
        with np.errstate(invalid="ignore"):
            ref = coef * h
        close(v, ref, (U[names[v.dtype]] + 8 * U32) * np.abs(ref) + TINY[names[v.dtype]], "clipped")
        assert bool((o[:3] == 7.0).all()) and bool((o[3 + v.numel():] == 7.0).all())
    assert all((np.nan_to_num(f64(g), nan=1.25) == np.nan_to_num(h, nan=1.25)).all() for g, h in zip(grads, host))
    dmt.dmt_grad_clip(lst, max_norm, None, ws)
    for g, v in zip(grads, views):
        assert torch.equal(g.nan_to_num(1.25), v.nan_to_num(1.25)), "in place, other values"


@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("count", [1, 2, 7, 60, 119, 120, 121, 250, 400])
def test_clip(dmt, count, shift):
    rng = np.random.default_rng(count)
    sizes = [int(s) for s in np.exp(rng.uniform(0, np.log(40_000), count))]
    sizes[0] = 100_003
    if count > 2:
        sizes[1], sizes[-1] = 0, 0
    kinds = [("f32", "f16", "bf16")[i % 3] for i in range(count)]
    for max_norm in (1.0, 1e9, 0.0):
        check_clip(dmt, grads_of(rng, sizes, kinds, shift, 0.1), max_norm)


@pytest.mark.parametrize("count", [133, 134, 135, 187, 188, 189, 269, 377])
def test_clip_of_as_many_as_a_launch_holds(dmt, count):
    test_clip(dmt, count, 1)


@pytest.mark.parametrize("n", [1, 7, 8, 9, 2047, 2048, 2049, 8192, 16_383, 16_384, 16_385, 32_767, 32_768, 32_769, 65_536,
                               65_537, 1_000_003, 9_000_001])
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_clip_of_one_tensor(dmt, n, kind):
    rng = np.random.default_rng(n)
    check_clip(dmt, grads_of(rng, [n], [kind], 1), 0.5)


def test_clip_of_nothing(dmt):
    got = torch.full((1,), 7.0, device="cuda")
    ws = bytes_buf(256)
    for grads in ([], [torch.empty(0, device="cuda")]):
        got.fill_(7.0)
        dmt.dmt_grad_norm(dmt.make_grad_list(grads), got, ws)
        assert float(got) == 0.0
        got.fill_(7.0)
        dmt.dmt_grad_clip(dmt.make_grad_list(grads), 1.0, got, ws)
        assert float(got) == 0.0


def test_clip_where_float32_squares_overflow_or_vanish(dmt):
    rng = np.random.default_rng(1)
    check_clip(dmt, grads_of(rng, [5000, 10], ["f32", "f32"], 0, 1e25), 1.0)
    check_clip(dmt, grads_of(rng, [5000, 10], ["bf16", "f32"], 0, 1e-30), 1e-32)
    check_clip(dmt, grads_of(rng, [5000], ["f32"], 0, 3e37), 1.0)            # the norm itself is beyond float32


def test_clip_of_gradients_that_are_not_finite(dmt):
    rng = np.random.default_rng(2)
    for value in (math.nan, math.inf, -math.inf):
        grads = grads_of(rng, [300, 40], ["f32", "bf16"])
        grads[1][7] = value
        check_clip(dmt, grads, 1.0)


# ------------------------------------------------------------------ streams and graphs


def _whole(dmt, seed):
    """Every entry point once: the inputs, the outputs, and the calls."""
    rng = np.random.default_rng(seed)
    n, rows, cols, vocab = 500, 300, 96, 5000
    s = dict(table=matrix(rng, rows, cols, "bf16"), ids=torch.from_numpy(some_ids(rng, n, rows, "holes")).cuda(),
             gamma=matrix(rng, 1, cols, "bf16")[0].contiguous(), beta=matrix(rng, 1, cols, "bf16")[0].contiguous(),
             dy=matrix(rng, n, cols, "f32"), x=matrix(rng, 20, vocab, "f16", scale=2.0),
             t=torch.from_numpy(rng.integers(0, vocab, 20).astype(np.int32)).cuda(), gl=matrix(rng, 1, 20, "f32")[0].contiguous())
    e = lambda *sh, dt=torch.float32: torch.zeros(*sh, dtype=dt, device="cuda")
    o = dict(emb=e(n, cols, dt=torch.bfloat16), y=e(n, cols, dt=torch.bfloat16), mean=e(n), rstd=e(n), dx=e(n, cols),
             dg=e(cols), db=e(cols), dtab=e(rows, cols), lp=e(20), h=e(20), st=e(20, 2), top=e(20, 10, dt=torch.int32),
             tlp=e(20, 10), dxs=e(20, vocab, dt=torch.float16), norm=e(1), cdg=e(cols), cdtab=e(rows, cols))
    ws = [bytes_buf(dmt.dmt_embed_bwd_workspace_bytes(n, rows, cols)), bytes_buf(dmt.dmt_layer_norm_bwd_workspace_bytes(n, cols)),
          bytes_buf(dmt.dmt_token_logprob_workspace_bytes(20, vocab, 10))]
    lst = dmt.make_grad_list([o["dg"], o["dtab"]], [o["cdg"], o["cdtab"]])
    ws.append(bytes_buf(dmt.dmt_grad_norm_workspace_bytes(lst)))

    def calls(stream=None):
        dmt.dmt_embed_fwd(s["table"], s["ids"], o["emb"], 3.0, stream=stream)
        dmt.dmt_layer_norm_fwd(o["emb"], s["gamma"], s["beta"], 1e-5, o["y"], o["mean"], o["rstd"], stream=stream)
        dmt.dmt_layer_norm_bwd(o["emb"], s["gamma"], o["mean"], o["rstd"], s["dy"], o["dx"], o["dg"], o["db"], ws[1], stream=stream)
        dmt.dmt_embed_bwd(s["ids"], o["dx"], o["dtab"], ws[0], 3.0, stream=stream)
        dmt.dmt_token_logprob_fwd(s["x"], s["t"], o["lp"], o["h"], o["top"], o["tlp"], o["st"], ws[2], stream=stream)
        dmt.dmt_token_logprob_bwd(s["x"], s["t"], o["st"], o["h"], s["gl"], s["gl"], o["dxs"], stream=stream)
        dmt.dmt_grad_clip(lst, 0.1, o["norm"], ws[3], stream=stream)

    return s, o, calls


def test_another_stream_and_a_graph_give_the_same(dmt):
    s, o, calls = _whole(dmt, 1)
    s2, o2, _ = _whole(dmt, 2)
    calls()
    torch.cuda.synchronize()
    first = {k: v.clone() for k, v in o.items()}
    side = torch.cuda.Stream()
    for v in o.values():
        v.zero_()
    side.wait_stream(torch.cuda.current_stream())
    calls(side)
    side.synchronize()
    assert all(torch.equal(first[k], o[k]) for k in o), [k for k in o if not torch.equal(first[k], o[k])]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(torch.cuda.current_stream())
    kept = {k: v.clone() for k, v in s.items()}
    for turn in range(4):                                # other inputs, then the first ones again
        src = s2 if turn % 2 else kept
        for k in s:
            s[k].copy_(src[k])
        for v in o.values():
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        by_graph = {k: v.clone() for k, v in o.items()}
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(by_graph[k], o[k]) for k in o), (turn, [k for k in o if not torch.equal(by_graph[k], o[k])])
        if turn % 2 == 0:
            assert all(torch.equal(first[k], o[k]) for k in o)
