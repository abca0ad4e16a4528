"""The sequence branch's oracle: its gradients against differences of its forward passes, and its edges."""
import numpy as np

from oracle import sequence as sq


def _difference(f, x, at, eps=1e-6):
    a, b = x.copy(), x.copy()
    a[at] += eps
    b[at] -= eps
    return (f(a) - f(b)) / (2 * eps)


def test_layer_norm_gradients_are_the_differences():
    rng = np.random.default_rng(0)
    x, dy = rng.normal(size=(3, 7)), rng.normal(size=(3, 7))
    gamma, beta = rng.normal(size=7), rng.normal(size=7)
    loss = lambda x, g, b: float((sq.layer_norm_fwd(x, g, b, 1e-5)[0] * dy).sum())
    _, mean, rstd = sq.layer_norm_fwd(x, gamma, beta, 1e-5)
    dx, dg, db = sq.layer_norm_bwd(x, gamma, mean, rstd, dy)
    for at in np.ndindex(3, 7):
        assert abs(_difference(lambda v: loss(v, gamma, beta), x, at) - dx[at]) < 1e-7
    for c in range(7):
        assert abs(_difference(lambda v: loss(x, v, beta), gamma, c) - dg[c]) < 1e-7
        assert abs(_difference(lambda v: loss(x, gamma, v), beta, c) - db[c]) < 1e-7


def test_token_logprob_gradient_is_the_difference():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(4, 9)) * 2
    x[1, 3] = x[2, 0] = -np.inf
    t = np.array([2, 4, -1, 8])
    gl, gh = rng.normal(size=4), rng.normal(size=4)

    def loss(v):
        lp, h, _, _ = sq.token_logprob(v, t, 0)
        return float((lp * gl + h * gh).sum())

    dx, _ = sq.token_logprob_bwd(x, t, gl, gh)
    for at in np.ndindex(4, 9):
        if x[at] > -np.inf:
            assert abs(_difference(loss, x, at) - dx[at]) < 1e-7, at
        else:
            assert dx[at] == 0


def test_embed_gradient_is_the_adjoint():
    rng = np.random.default_rng(2)
    table, ids = rng.normal(size=(5, 3)), np.array([0, 4, 4, -1, 2, 5, 4])
    g = rng.normal(size=(7, 3))
    d, size = sq.embed_bwd(ids, g, 5, 1.5)
    assert abs((sq.embed_fwd(table, ids, 1.5) * g).sum() - (table * d).sum()) < 1e-12
    assert (d[[1, 3]] == 0).all() and (size >= np.abs(d) - 1e-15).all()


def test_rows_that_hold_nothing_and_ties():
    x = np.array([[-np.inf, -np.inf, -np.inf], [1.0, 1.0, -np.inf], [0.0, -0.0, 0.0]])
    lp, h, ids, lps = sq.token_logprob(x, np.array([1, 0, -1]), 3)
    assert lp[0] == -np.inf and h[0] == 0 and (ids[0] == -1).all()
    assert ids[1].tolist() == [0, 1, -1] and lps[1, 2] == -np.inf and abs(h[1] - np.log(2)) < 1e-15
    assert ids[2].tolist() == [0, 1, 2] and lp[2] == 0
    assert sq.grad_clip([np.array([3.0]), np.array([4.0])], 1.0)[0] == 5.0
