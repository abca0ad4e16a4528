"""What the sequence branch's entry points refuse, from the host checks alone (nothing is launched)."""
import ctypes

import pytest

import paper_2403_00877_amd as dmt
from paper_2403_00877_amd import binding

OK, EINVAL, ENOTSUP, ENOMEM = binding.DMT_OK, binding.DMT_EINVAL, binding.DMT_ENOTSUP, binding.DMT_ENOMEM
lib = binding._lib
P, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4098)


def call(name, order, defaults, **kw):
    assert set(kw) <= set(defaults), kw
    a = dict(defaults, **kw)
    return getattr(lib, name)(*[a[k] for k in order.split()])


EMBED_FWD = ("dmt_embed_fwd", "table rows cols ts td ids n scale out os od bad stream",
             dict(table=P, rows=10, cols=8, ts=8, td=2, ids=P, n=4, scale=1.0, out=P, os=8, od=2, bad=None, stream=None))
EMBED_BWD = ("dmt_embed_bwd", "ids n grad gs gd scale out rows cols os acc bad ws wsb stream",
             dict(ids=P, n=4, grad=P, gs=8, gd=2, scale=1.0, out=P, rows=10, cols=8, os=8, acc=0, bad=None, ws=P,
                  wsb=1 << 30, stream=None))
NORM_FWD = ("dmt_layer_norm_fwd", "x rows cols xs dt gamma beta wd eps y ys mean rstd stream",
            dict(x=P, rows=4, cols=8, xs=8, dt=2, gamma=P, beta=P, wd=0, eps=1e-5, y=P, ys=8, mean=None, rstd=None,
                 stream=None))
NORM_BWD = ("dmt_layer_norm_bwd", "x rows cols xs dt gamma wd mean rstd dy dys gd dx dxs dgamma dbeta ws wsb stream",
            dict(x=P, rows=4, cols=8, xs=8, dt=2, gamma=P, wd=0, mean=P, rstd=P, dy=P, dys=8, gd=0, dx=P, dxs=8,
                 dgamma=P, dbeta=P, ws=P, wsb=1 << 30, stream=None))
LP_FWD = ("dmt_token_logprob_fwd", "x rows vocab xs dt targets lp h stats k ids tlp bad ws wsb stream",
          dict(x=P, rows=4, vocab=8, xs=8, dt=2, targets=P, lp=P, h=P, stats=P, k=2, ids=P, tlp=P, bad=None, ws=P,
               wsb=1 << 30, stream=None))
LP_BWD = ("dmt_token_logprob_bwd", "x rows vocab xs dt targets stats h gl gh dx dxs stream",
          dict(x=P, rows=4, vocab=8, xs=8, dt=2, targets=P, stats=P, h=P, gl=P, gh=P, dx=P, dxs=8, stream=None))


@pytest.mark.parametrize("kw,code", [
    (dict(rows=0), EINVAL), (dict(cols=0), EINVAL), (dict(n=-1), EINVAL), (dict(ts=7), EINVAL), (dict(os=7), EINVAL),
    (dict(td=3), EINVAL), (dict(od=-1), EINVAL), (dict(table=None), EINVAL), (dict(ids=None), EINVAL),
    (dict(out=None), EINVAL), (dict(ids=ODD), EINVAL), (dict(td=0, table=ODD), EINVAL), (dict(od=0, out=ODD), EINVAL),
    (dict(bad=ctypes.c_void_p(4100)), EINVAL), (dict(n=1 << 31), ENOTSUP), (dict(rows=1 << 31), ENOTSUP),
    (dict(cols=(1 << 24) + 1, ts=1 << 25, os=1 << 25), ENOTSUP), (dict(n=0, ids=None, out=None), OK)])
def test_embed_fwd_refuses(kw, code):
    assert call(*EMBED_FWD, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(rows=0), EINVAL), (dict(cols=0), EINVAL), (dict(n=-1), EINVAL), (dict(gs=7), EINVAL), (dict(os=7), EINVAL),
    (dict(gd=3), EINVAL), (dict(grad=None), EINVAL), (dict(ids=None), EINVAL), (dict(out=None), EINVAL),
    (dict(out=ODD), EINVAL), (dict(gd=0, grad=ODD), EINVAL), (dict(ws=None), EINVAL),
    (dict(ws=ctypes.c_void_p(4160)), EINVAL), (dict(wsb=16), ENOMEM), (dict(n=1 << 31), ENOTSUP),
    (dict(bad=ODD), EINVAL)])
def test_embed_bwd_refuses(kw, code):
    assert call(*EMBED_BWD, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(xs=7), EINVAL), (dict(ys=7), EINVAL), (dict(dt=5), EINVAL),
    (dict(wd=1), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(x=None), EINVAL),
    (dict(y=None), EINVAL), (dict(gamma=ODD), EINVAL), (dict(mean=ODD), EINVAL), (dict(xs=9), EINVAL),   # in place, strides differ
    (dict(rows=1 << 31), ENOTSUP), (dict(cols=(1 << 24) + 1, xs=1 << 25, ys=1 << 25), ENOTSUP),
    (dict(rows=0, x=None, y=None), OK)])
def test_layer_norm_fwd_refuses(kw, code):
    assert call(*NORM_FWD, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(xs=7), EINVAL), (dict(dys=7), EINVAL), (dict(dxs=7), EINVAL),
    (dict(dt=5), EINVAL), (dict(wd=1), EINVAL), (dict(gd=1), EINVAL), (dict(x=None), EINVAL), (dict(dy=None), EINVAL),
    (dict(dx=None), EINVAL), (dict(mean=None), EINVAL), (dict(rstd=None), EINVAL), (dict(dgamma=ODD), EINVAL),
    (dict(dys=9), EINVAL), (dict(ws=None), EINVAL), (dict(wsb=16), ENOMEM), (dict(rows=1 << 31), ENOTSUP)])
def test_layer_norm_bwd_refuses(kw, code):
    assert call(*NORM_BWD, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), EINVAL), (dict(vocab=0), EINVAL), (dict(xs=7), EINVAL), (dict(dt=3), EINVAL), (dict(k=-1), EINVAL),
    (dict(k=65), EINVAL), (dict(x=None), EINVAL), (dict(targets=None), EINVAL), (dict(ids=None), EINVAL),
    (dict(lp=ODD), EINVAL), (dict(dt=0, x=ODD), EINVAL), (dict(rows=1 << 31), ENOTSUP),
    (dict(vocab=(1 << 30) + 1, xs=1 << 31), ENOTSUP), (dict(rows=0, x=None), OK)])
def test_token_logprob_fwd_refuses(kw, code):
    assert call(*LP_FWD, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), EINVAL), (dict(vocab=0), EINVAL), (dict(xs=7), EINVAL), (dict(dxs=7), EINVAL), (dict(dt=3), EINVAL),
    (dict(x=None), EINVAL), (dict(dx=None), EINVAL), (dict(stats=None), EINVAL), (dict(targets=None), EINVAL),
    (dict(h=None), EINVAL), (dict(dxs=9), EINVAL), (dict(rows=1 << 31), ENOTSUP), (dict(rows=0, x=None, dx=None), OK)])
def test_token_logprob_bwd_refuses(kw, code):
    assert call(*LP_BWD, **kw) == code


def _grads(*specs):
    arr = (binding.dmt_grad_tensor * max(1, len(specs)))()
    for a, s in zip(arr, specs):
        a.data, a.out, a.numel, a.dtype = s
    return arr


def test_grad_norm_and_clip_refuse():
    ws, big = ctypes.c_void_p(4096), 1 << 30
    norm = lambda arr, n, norm=P, ws=ws, b=big: lib.dmt_grad_norm(arr, n, norm, ws, b, None)
    clip = lambda arr, n, mx=1.0, norm=P, ws=ws, b=big: lib.dmt_grad_clip(arr, n, mx, norm, ws, b, None)
    good = _grads((4096, 4096, 10, 0))
    for f in (norm, clip):
        assert f(good, -1) == EINVAL and f(None, 1) == EINVAL and f(good, (1 << 20) + 1) == ENOTSUP
        assert f(_grads((None, 4096, 10, 0)), 1) == EINVAL
        assert f(_grads((4098, 4096, 10, 0)), 1) == EINVAL
        assert f(_grads((4096, 4096, -1, 0)), 1) == EINVAL
        assert f(_grads((4096, 4096, 10, 3)), 1) == EINVAL
        assert f(_grads((4096, 4096, (1 << 40) + 1, 0)), 1) == ENOTSUP
        assert f(good, 1, ws=None) == EINVAL and f(good, 1, b=4) == ENOMEM
    assert norm(good, 1, norm=None) == EINVAL
    assert clip(_grads((4096, None, 10, 0)), 1) == EINVAL
    assert clip(good, 1, mx=-1.0) == EINVAL and clip(good, 1, mx=float("nan")) == EINVAL
    assert lib.dmt_grad_norm_workspace_bytes(_grads((None, None, 0, 0)), 1) > 0


def test_workspaces_are_host_arithmetic():
    assert dmt.dmt_embed_bwd_workspace_bytes(0, 1, 1) >= 0
    assert dmt.dmt_embed_bwd_workspace_bytes(1000, 100, 8) >= 8000
    assert dmt.dmt_embed_bwd_workspace_bytes(-1, 100, 8) == 0
    assert dmt.dmt_layer_norm_bwd_workspace_bytes(0, 7) >= 0
    assert dmt.dmt_layer_norm_bwd_workspace_bytes(5, 0) == 0
    assert dmt.dmt_token_logprob_workspace_bytes(3, 100, 65) == 0
