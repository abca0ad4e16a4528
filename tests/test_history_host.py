"""What the history block's entry points refuse, from the host checks alone (nothing is launched)."""
import ctypes

import pytest

import paper_2403_00877_amd as dmt
from paper_2403_00877_amd import binding

OK, EINVAL, ENOTSUP, ENOMEM = binding.DMT_OK, binding.DMT_EINVAL, binding.DMT_ENOTSUP, binding.DMT_ENOMEM
lib = binding._lib
P, Q, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(8192), ctypes.c_void_p(4098)
BYTE = ctypes.c_void_p(4097)


def call(name, order, defaults, **kw):
    assert set(kw) <= set(defaults), kw
    a = dict(defaults, **kw)
    return getattr(lib, name)(*[a[k] for k in order.split()])


ROWS = ("dmt_sequence_rows", "off n rows out bad stream", dict(off=P, n=3, rows=9, out=P, bad=None, stream=None))
FWD = ("dmt_gated_scan_fwd", "g gs v vs rows cols dt form seq n init h hs fin kept kb bad ws wsb stream",
       dict(g=P, gs=8, v=P, vs=8, rows=4, cols=8, dt=2, form=0, seq=P, n=2, init=None, h=P, hs=8, fin=None, kept=P, kb=1 << 30,
            bad=None, ws=P, wsb=1 << 30, stream=None))
BWD = ("dmt_gated_scan_bwd", "g gs v vs rows cols dt form seq n init kept kb dh dhs gd df dg dgs dv dvs di ws wsb stream",
       dict(g=P, gs=8, v=P, vs=8, rows=4, cols=8, dt=2, form=1, seq=P, n=2, init=None, kept=P, kb=1 << 30, dh=P, dhs=8, gd=0,
            df=None, dg=P, dgs=8, dv=P, dvs=8, di=None, ws=P, wsb=1 << 30, stream=None))
STEP = ("dmt_gated_scan_step", "g gs v vs rows cols dt form slots state new states h hs bad stream",
        dict(g=P, gs=8, v=P, vs=8, rows=4, cols=8, dt=2, form=0, slots=P, state=P, new=P, states=9, h=P, hs=8, bad=None,
             stream=None))
DROP = ("dmt_dropout_fwd", "x rows cols xs dt res rs p rng site y ys stream",
        dict(x=P, rows=4, cols=8, xs=8, dt=2, res=None, rs=0, p=0.5, rng=P, site=0, y=Q, ys=8, stream=None))
DROP_BWD = ("dmt_dropout_bwd", "x rows cols xs dt p rng site y ys stream",
            dict(x=P, rows=4, cols=8, xs=8, dt=2, p=0.5, rng=P, site=0, y=Q, ys=8, stream=None))
SORT = ("dmt_expert_sort", "e n k E cap slot src off cnt bad ws wsb stream",
        dict(e=P, n=4, k=2, E=8, cap=0, slot=P, src=P, off=P, cnt=P, bad=None, ws=P, wsb=1 << 30, stream=None))
GATHER = ("dmt_expert_gather", "x n cols xs dt slot k src rows out os stream",
          dict(x=P, n=4, cols=8, xs=8, dt=2, slot=P, k=2, src=P, rows=8, out=Q, os=8, stream=None))
COMBINE = ("dmt_expert_combine", "z rows cols zs dt slot n k w y ys yd stream",
           dict(z=P, rows=8, cols=8, zs=8, dt=2, slot=P, n=4, k=2, w=P, y=Q, ys=8, yd=2, stream=None))
COMBINE_BWD = ("dmt_expert_combine_bwd", "dy n cols dys gd z rows zs dt slot k src w dz dzs dw stream",
               dict(dy=P, n=4, cols=8, dys=8, gd=0, z=P, rows=8, zs=8, dt=2, slot=P, k=2, src=P, w=P, dz=Q, dzs=8, dw=P,
                    stream=None))
LARGE = (1 << 30) + 1
WIDE = (1 << 24) + 1


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(off=None), EINVAL), (dict(off=ctypes.c_void_p(4100)), EINVAL),
    (dict(out=None), EINVAL), (dict(out=ODD), EINVAL), (dict(bad=ctypes.c_void_p(4100)), EINVAL), (dict(rows=LARGE), ENOTSUP),
    (dict(n=LARGE), ENOTSUP), (dict(n=0, rows=0, out=None), OK)])
def test_sequence_rows_refuses(kw, code):
    assert call(*ROWS, **kw) == code


SCAN = [(dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(n=-1), EINVAL), (dict(gs=7), EINVAL), (dict(vs=7), EINVAL),
        (dict(dt=3), EINVAL), (dict(form=2), EINVAL), (dict(form=-1), EINVAL), (dict(g=None), EINVAL), (dict(v=None), EINVAL),
        (dict(g=BYTE), EINVAL), (dict(seq=ODD), EINVAL), (dict(init=ODD), EINVAL), (dict(seq=None, n=3), EINVAL),
        (dict(seq=None, n=0), EINVAL), (dict(rows=LARGE), ENOTSUP), (dict(n=LARGE), ENOTSUP), (dict(kb=3), ENOMEM),
        (dict(cols=WIDE, gs=WIDE, vs=WIDE, hs=WIDE, dhs=WIDE, dgs=WIDE, dvs=WIDE), ENOTSUP),
        (dict(rows=10 ** 6, wsb=64), ENOMEM), (dict(rows=10 ** 6, ws=None), EINVAL), (dict(rows=10 ** 6, ws=ctypes.c_void_p(4160)), EINVAL),
        (dict(kept=ctypes.c_void_p(4160)), EINVAL)]


@pytest.mark.parametrize("kw,code", SCAN + [
    (dict(hs=7), EINVAL), (dict(h=None), EINVAL), (dict(fin=ODD), EINVAL), (dict(fin=Q, init=Q), EINVAL),
    (dict(bad=ctypes.c_void_p(4100)), EINVAL), (dict(rows=0, g=None, v=None, h=None, seq=None, n=0, ws=None, wsb=0), OK)])
def test_gated_scan_fwd_refuses(kw, code):
    known = {k: v for k, v in kw.items() if k in FWD[2]}
    assert call(*FWD, **known) == code


@pytest.mark.parametrize("kw,code", SCAN + [
    (dict(dhs=7), EINVAL), (dict(dgs=7), EINVAL), (dict(dvs=7), EINVAL), (dict(gd=1), EINVAL), (dict(dh=None), EINVAL),
    (dict(dg=None), EINVAL), (dict(dv=None), EINVAL), (dict(dh=ODD), EINVAL), (dict(kept=None), EINVAL), (dict(df=ODD), EINVAL),
    (dict(di=ODD), EINVAL), (dict(df=Q, di=Q), EINVAL),
    (dict(rows=0, g=None, v=None, dh=None, dg=None, dv=None, kept=None, kb=0, ws=None, wsb=0), OK)])
def test_gated_scan_bwd_refuses(kw, code):
    known = {k: v for k, v in kw.items() if k in BWD[2]}
    assert call(*BWD, **known) == code


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(states=-1), EINVAL), (dict(gs=7), EINVAL), (dict(vs=7), EINVAL),
    (dict(hs=7), EINVAL), (dict(dt=4), EINVAL), (dict(form=5), EINVAL), (dict(g=None), EINVAL), (dict(v=None), EINVAL),
    (dict(h=None), EINVAL), (dict(state=None), EINVAL), (dict(new=None), EINVAL), (dict(new=ODD), EINVAL),
    (dict(slots=ODD), EINVAL), (dict(slots=None, states=3), EINVAL), (dict(rows=65537), ENOTSUP),
    (dict(states=LARGE), ENOTSUP), (dict(cols=WIDE, gs=WIDE, vs=WIDE, hs=WIDE), ENOTSUP),
    (dict(rows=0, g=None, v=None, h=None), OK)])
def test_gated_scan_step_refuses(kw, code):
    assert call(*STEP, **kw) == code


DROPS = [(dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(xs=7), EINVAL), (dict(ys=7), EINVAL), (dict(dt=3), EINVAL),
         (dict(p=-0.1), EINVAL), (dict(p=1.1), EINVAL), (dict(p=float("nan")), EINVAL), (dict(site=-1), EINVAL),
         (dict(site=2048), EINVAL), (dict(rng=None), EINVAL), (dict(rng=ctypes.c_void_p(4100)), EINVAL), (dict(x=None), EINVAL),
         (dict(y=None), EINVAL), (dict(x=BYTE), EINVAL), (dict(y=P, ys=9), EINVAL), (dict(rows=1 << 31), ENOTSUP),
         (dict(cols=WIDE, xs=WIDE, ys=WIDE), ENOTSUP), (dict(rows=0, x=None, y=None), OK)]


@pytest.mark.parametrize("kw,code", DROPS + [(dict(res=P, rs=7), EINVAL), (dict(res=BYTE, rs=8), EINVAL),
                                             (dict(res=Q, rs=9), EINVAL)])
def test_dropout_fwd_refuses(kw, code):
    assert call(*DROP, **kw) == code


@pytest.mark.parametrize("kw,code", DROPS)
def test_dropout_bwd_refuses(kw, code):
    assert call(*DROP_BWD, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), EINVAL), (dict(k=0), EINVAL), (dict(E=0), EINVAL), (dict(cap=-1), EINVAL), (dict(e=None), EINVAL),
    (dict(slot=None), EINVAL), (dict(src=None), EINVAL), (dict(e=ODD), EINVAL), (dict(off=ODD), EINVAL), (dict(cnt=ODD), EINVAL),
    (dict(E=1025), ENOTSUP), (dict(n=1 << 30), ENOTSUP), (dict(k=1 << 40), ENOTSUP), (dict(cap=1 << 28), ENOTSUP),
    (dict(n=10 ** 6, wsb=16), ENOMEM), (dict(n=10 ** 6, ws=None), EINVAL), (dict(bad=ctypes.c_void_p(4100)), EINVAL)])
def test_expert_sort_refuses(kw, code):
    assert call(*SORT, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(k=0), EINVAL), (dict(xs=7), EINVAL),
    (dict(os=7), EINVAL), (dict(dt=3), EINVAL), (dict(x=None), EINVAL), (dict(slot=None), EINVAL), (dict(src=None), EINVAL),
    (dict(out=None), EINVAL), (dict(x=BYTE), EINVAL), (dict(rows=1 << 31), ENOTSUP), (dict(n=1 << 30), ENOTSUP),
    (dict(cols=WIDE, xs=WIDE, os=WIDE), ENOTSUP), (dict(rows=0, n=0, x=None, slot=None, src=None, out=None), OK)])
def test_expert_gather_refuses(kw, code):
    assert call(*GATHER, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(k=0), EINVAL), (dict(zs=7), EINVAL),
    (dict(ys=7), EINVAL), (dict(dt=3), EINVAL), (dict(yd=-1), EINVAL), (dict(z=None), EINVAL), (dict(y=None), EINVAL),
    (dict(slot=None), EINVAL), (dict(w=ODD), EINVAL), (dict(yd=0, y=ODD), EINVAL), (dict(n=1 << 30), ENOTSUP),
    (dict(rows=1 << 31), ENOTSUP), (dict(cols=WIDE, zs=WIDE, ys=WIDE), ENOTSUP), (dict(n=0, slot=None, y=None), OK)])
def test_expert_combine_refuses(kw, code):
    assert call(*COMBINE, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(k=0), EINVAL), (dict(dys=7), EINVAL),
    (dict(zs=7), EINVAL), (dict(dzs=7), EINVAL), (dict(dt=3), EINVAL), (dict(gd=1), EINVAL), (dict(dy=None), EINVAL),
    (dict(z=None), EINVAL), (dict(src=None), EINVAL), (dict(slot=None), EINVAL), (dict(dz=ODD), EINVAL), (dict(dw=ODD), EINVAL),
    (dict(w=ODD), EINVAL), (dict(n=1 << 30), ENOTSUP), (dict(rows=1 << 31), ENOTSUP),
    (dict(cols=WIDE, zs=WIDE, dys=WIDE, dzs=WIDE), ENOTSUP),
    (dict(n=0, rows=0, dy=None, z=None, slot=None, src=None), OK)])
def test_expert_combine_bwd_refuses(kw, code):
    assert call(*COMBINE_BWD, **kw) == code


def test_workspaces_are_host_arithmetic():
    assert dmt.dmt_gated_scan_workspace_bytes(0, 5) == 0 and dmt.dmt_gated_scan_workspace_bytes(-1, 5) == 0
    assert dmt.dmt_gated_scan_workspace_bytes(10 ** 6, 64) > 0 and dmt.dmt_gated_scan_workspace_bytes(LARGE, 1) == 0
    assert dmt.dmt_gated_scan_kept_bytes(17, 3) == 36 and dmt.dmt_gated_scan_kept_bytes(0, 3) == 0
    assert dmt.dmt_expert_sort_workspace_bytes(10, 2, 8) == 0 and dmt.dmt_expert_sort_workspace_bytes(10 ** 6, 2, 8) > 0
    assert dmt.dmt_expert_sort_workspace_bytes(10 ** 6, 2, 1025) == 0
