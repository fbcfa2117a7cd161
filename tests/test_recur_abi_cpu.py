"""Host-side refusals of the recurrence's entry points (nothing is launched, no GPU needed)."""

import ctypes as C

import pytest
import torch

from paper_2111_05188_amd import tp

X = 0x100000


def _cfg(T=4, B=3, D=8, dtype=tp.TP_F32):
    return tp.Recur(T, B, D, dtype, X, None, None)


def _rows(c, p=X, st=None, sb=None):
    return C.byref(tp.Rows(p, c.B * c.D if st is None else st, c.D if sb is None else sb))


def _forward(c, **kw):
    L = tp.load()
    r = _rows(c)
    a = dict(cfg=C.byref(c), x=r, r=r, i=r, h0=None, y=r, h_last=None, saved=None, work=X,
             nb=1 << 30, stream=None)
    a.update(kw)
    return L.tp_recur_forward(*a.values())


def _backward(c, **kw):
    L = tp.load()
    r = _rows(c)
    a = dict(cfg=C.byref(c), x=r, r=r, i=r, saved=X, dy=r, dh_last=None, dx=r, dr=r, di=r, dlam=X,
             dh0=None, work=X, nb=1 << 30, stream=None)
    a.update(kw)
    return L.tp_recur_backward(*a.values())


def _refused(rc, text, code=tp.TP_EINVAL):
    assert rc == code and text in tp.last_error(), (rc, tp.last_error())


def test_sizes():
    L = tp.load()
    c = _cfg(T=17)
    assert L.tp_recur_saved_bytes(C.byref(c)) == 3 * 3 * 8 * 4      # states before steps 0, 8, 16
    assert L.tp_recur_workspace_bytes(C.byref(c)) >= 256
    for bad in (dict(T=0), dict(B=0), dict(D=0), dict(T=-1), dict(dtype=7)):
        assert L.tp_recur_saved_bytes(C.byref(_cfg(**bad))) == 0
        assert L.tp_recur_workspace_bytes(C.byref(_cfg(**bad))) == 0
        _refused(_forward(_cfg(**bad)), "recurrence")
    assert L.tp_recur_workspace_bytes(None) == 0
    _refused(_forward(_cfg(B=1 << 30, D=64)), "grid", tp.TP_EUNSUPPORTED)
    _refused(_forward(_cfg(B=1, D=(1 << 24) + 1)), "grid", tp.TP_EUNSUPPORTED)
    _refused(_forward(_cfg(T=(1 << 30) + 1, B=1, D=1)), "grid", tp.TP_EUNSUPPORTED)


def test_forward_refuses():
    c = _cfg()
    _refused(_forward(c, cfg=None), "NULL")
    _refused(_forward(c, x=None), "x is NULL")
    _refused(_forward(c, r=C.byref(tp.Rows(None, 0, 0))), "r is NULL")
    _refused(_forward(c, i=_rows(c, X + 2)), "i is misaligned")
    _refused(_forward(c, x=_rows(c, st=-1)), "strides")
    _refused(_forward(c, work=None), "workspace")
    _refused(_forward(c, work=X + 8), "workspace")
    _refused(_forward(c, nb=0), "needed")
    _refused(_forward(c, y=None), "no output")
    _refused(_forward(c, h0=X + 1), "misaligned")
    for st, sb in ((0, 8), (24, 7), (8, 8), (16, 8), (8, 31)):
        _refused(_forward(c, y=_rows(c, st=st, sb=sb)), "overlap")
    c.lam = None
    _refused(_forward(c), "lambda")


def test_backward_refuses():
    c = _cfg()
    for k in ("x", "dy", "dx", "dr", "di"):
        _refused(_backward(c, **{k: None}), f"{k} is NULL")
    _refused(_backward(c, saved=None), "saved")
    _refused(_backward(c, dlam=None), "dlambda")
    _refused(_backward(c, di=_rows(c, sb=4)), "overlap")
    _refused(_backward(c, nb=1), "needed")


def test_step_refuses():
    L = tp.load()
    c = _cfg(T=1)
    r = _rows(c)
    ok = dict(cfg=C.byref(c), x=r, r=r, i=r, h=X, h_out=X, y=r, stream=None)

    def step(**kw):
        return L.tp_recur_step(*{**ok, **kw}.values())

    _refused(step(cfg=C.byref(_cfg(T=2))), "must be 1")
    _refused(step(cfg=C.byref(tp.Recur(1, 3, 8, tp.TP_F32, X, None, X))), "len")
    _refused(step(h=None), "state")
    _refused(step(h_out=X + 2), "state")
    _refused(step(x=None), "x is NULL")
    _refused(step(y=_rows(c, sb=3)), "overlap")


def test_states_that_overlap_in_part_are_refused():
    c = _cfg()
    _refused(_forward(c, h0=X, h_last=X + 4), "h0 and h_last")
    _refused(_forward(c, h0=X + 4 * (3 * 8 - 1), h_last=X), "h0 and h_last")
    _refused(_backward(c, dh_last=X, dh0=X + 4), "dh_last and dh0")
    L, c = tp.load(), _cfg(T=1)
    r = _rows(c)
    _refused(L.tp_recur_step(C.byref(c), r, r, r, X, X + 32, r, None), "h and h_out")


def test_kept_states_of_another_type_or_without_memory_are_refused():
    """As many elements, but fewer bytes than the kernels write."""
    T, B, D = 40, 3, 8
    rc = tp.RecurT(torch.zeros(D), T, B, torch.float32)
    x, n = torch.zeros(T, B, D), rc.saved_count
    work, dlam = rc.workspace(), torch.zeros(D)
    for saved in (torch.zeros(n, dtype=torch.bfloat16), torch.zeros(n, dtype=torch.uint8),
                  torch.zeros(1).expand(n), torch.zeros(n - 1)):
        with pytest.raises(AssertionError):
            tp.recur_forward(rc, x, x, x, x.clone(), work, saved=saved)
        with pytest.raises(AssertionError):
            tp.recur_backward(rc, x, x, x, saved, x, x, x, x, dlam, work)
    with pytest.raises(AssertionError):
        tp.recur_forward(rc, x, x, x, x.clone(), work[:1].expand(work.numel()))
