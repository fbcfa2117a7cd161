"""Host-side refusals of the delta rule's entry points (nothing is launched, no GPU needed)."""

import ctypes as C

import pytest
import torch

from paper_2111_05188_amd import tp

X = 0x100000


def _cfg(T=4, B=3, H=2, dk=8, dv=6, dtype=tp.TP_F32):
    return tp.Delta(T, B, H, dk, dv, dtype, X, None, None)


def _heads(c, d, p=X, st=None, sb=None, sh=None):
    return C.byref(tp.Heads(p, c.B * c.H * d if st is None else st, c.H * d if sb is None else sb,
                            d if sh is None else sh))


def _inputs(c):
    return dict(q=_heads(c, c.dk), k=_heads(c, c.dk), v=_heads(c, c.dv), r=_heads(c, 1),
                b=_heads(c, 1))


def _forward(c, **kw):
    a = dict(cfg=C.byref(c), **_inputs(c), h0=None, y=_heads(c, c.dv), h_last=None, saved=None,
             work=X, nb=1 << 30, stream=None)
    a.update(kw)
    return tp.load().tp_delta_forward(*a.values())


def _backward(c, **kw):
    out = {"d" + k: v for k, v in _inputs(c).items()}
    a = dict(cfg=C.byref(c), **_inputs(c), saved=X, dy=_heads(c, c.dv), dh_last=None, **out,
             dlam=X, dh0=None, work=X, nb=1 << 30, stream=None)
    a.update(kw)
    return tp.load().tp_delta_backward(*a.values())


def _step(c, **kw):
    a = dict(cfg=C.byref(c), **_inputs(c), h=X, h_out=X, y=_heads(c, c.dv), stream=None)
    a.update(kw)
    return tp.load().tp_delta_step(*a.values())


def _refused(rc, text, code=tp.TP_EINVAL):
    assert rc == code and text in tp.last_error(), (rc, tp.last_error())


def test_sizes():
    L = tp.load()
    c = _cfg(T=33)
    assert L.tp_delta_saved_bytes(C.byref(c)) >= 3 * 2 * 8 * 6 * 4
    assert L.tp_delta_saved_bytes(C.byref(c)) % 16 == 0
    assert L.tp_delta_workspace_bytes(C.byref(c)) >= 256
    for bad in (dict(T=0), dict(B=0), dict(H=0), dict(dk=0), dict(dv=-1), dict(dtype=7)):
        assert L.tp_delta_saved_bytes(C.byref(_cfg(**bad))) == 0
        assert L.tp_delta_workspace_bytes(C.byref(_cfg(**bad))) == 0
        _refused(_forward(_cfg(**bad)), "delta rule")
    assert L.tp_delta_workspace_bytes(None) == 0
    for bad, text in ((dict(dk=129), "at most 128"), (dict(dv=129), "at most 128"),
                      (dict(B=1 << 22, H=4), "grid"), (dict(T=(1 << 30) + 1), "grid")):
        _refused(_forward(_cfg(**bad)), text, tp.TP_EUNSUPPORTED)


def test_forward_refuses():
    c = _cfg()
    _refused(_forward(c, cfg=None), "NULL")
    for name in "qkvrb":
        _refused(_forward(c, **{name: None}), f"{name} is NULL")
        _refused(_forward(c, **{name: _heads(c, 8, X + 2)}), f"{name} is misaligned")
        _refused(_forward(c, **{name: _heads(c, 8, st=-1)}), "strides")
        _refused(_forward(c, **{name: _heads(c, 8, sh=(1 << 40) + 1)}), "strides")
    _refused(_forward(c, work=None), "workspace")
    _refused(_forward(c, work=X + 8), "workspace")
    _refused(_forward(c, nb=0), "needed")
    _refused(_forward(c, y=None), "no output")
    _refused(_forward(c, h0=X + 1), "misaligned")
    _refused(_forward(c, saved=X + 4), "16-byte")
    # rows of 6: heads, sequences or steps on one another
    for st, sb, sh in ((36, 12, 5), (36, 11, 6), (35, 12, 6), (0, 12, 6), (6, 24, 6), (12, 48, 7),
                       (24, 24, 6)):
        _refused(_forward(c, y=_heads(c, 6, st=st, sb=sb, sh=sh)), "overlap")
    # any order of the axes is allowed, and a state in the place of the other
    for bad in (dict(h0=X, h_last=X + 4), dict(h0=X + 4 * (3 * 2 * 48 - 1), h_last=X)):
        _refused(_forward(c, **bad), "h0 and h_last")
    c.lam = None
    _refused(_forward(c), "lambda")


def test_backward_refuses():
    c = _cfg()
    for name in ("q", "dy", "dq", "dk", "dv", "dr", "db"):
        _refused(_backward(c, **{name: None}), f"{name} is NULL")
    for name in ("dq", "dk", "dv"):
        _refused(_backward(c, **{name: _heads(c, 8, sh=3)}), "overlap")
    _refused(_backward(c, dr=_heads(c, 1, sh=0)), "overlap")
    _refused(_backward(c, saved=None), "saved")
    _refused(_backward(c, saved=X + 4), "misaligned")
    _refused(_backward(c, dlam=None), "dlambda")
    _refused(_backward(c, nb=1), "needed")
    _refused(_backward(c, dh_last=X, dh0=X + 4), "dh_last and dh0")


def test_step_refuses():
    c = _cfg(T=1)
    _refused(_step(_cfg(T=2)), "must be 1")
    _refused(_step(tp.Delta(1, 3, 2, 8, 6, tp.TP_F32, X, None, X)), "len")
    _refused(_step(c, h=None), "state")
    _refused(_step(c, h_out=X + 2), "state")
    _refused(_step(c, h_out=X + 64), "h and h_out")
    _refused(_step(c, q=None), "q is NULL")
    _refused(_step(c, y=_heads(c, 6, sh=5)), "overlap")


def test_the_binding_checks_shapes_and_types():
    T, B, H, dk, dv = 5, 3, 2, 8, 6
    dc = tp.DeltaT(torch.zeros(H), T, B, dk, dv, torch.float32)
    q, v, r = torch.zeros(T, B, H, dk), torch.zeros(T, B, H, dv), torch.zeros(T, B, H)
    work, n, dlam = dc.workspace(), dc.saved_count, torch.zeros(H)
    for bad in ((q, q, q, r, r), (q, v, v, r, r), (q, q, v, q, r), (q.bfloat16(), q, v, r, r),
                (q.transpose(0, 3).contiguous().transpose(0, 3), q, v, r, r)):
        with pytest.raises(AssertionError):
            tp.delta_forward(dc, *bad, v.clone(), work)
    for saved in (torch.zeros(n, dtype=torch.bfloat16), torch.zeros(1).expand(n), torch.zeros(n - 1)):
        with pytest.raises(AssertionError):
            tp.delta_forward(dc, q, q, v, r, r, v.clone(), work, saved=saved)
        with pytest.raises(AssertionError):
            tp.delta_backward(dc, q, q, v, r, r, saved, v, q, q, v, r, r, dlam, work)
    h = torch.zeros(B, H, dk, dv)
    with pytest.raises(AssertionError):
        tp.delta_step(q[0], q[0], v[0], r[0], r[0], torch.zeros(H), h, h.bfloat16())
    with pytest.raises(AssertionError):
        tp.delta_step(q[0], q[0], v[0], r[0], r[0], torch.zeros(H + 1), h, h)
    with pytest.raises(tp.TPError):
        tp.DeltaT(torch.zeros(H), T, B, 129, dv, torch.float32)


def test_the_launch_grid_is_not_overrun():
    """2^23 heads of 128 channels would be 2^32 threads."""
    for B, H in ((1 << 23, 1), (1 << 20, 8)):
        _refused(_forward(_cfg(T=1, B=B, H=H)), "grid", tp.TP_EUNSUPPORTED)
