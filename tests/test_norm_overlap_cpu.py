"""Arrays of the norms that overlap: refused on the host, before anything is launched."""

import ctypes as C

import pytest

from paper_2111_05188_amd import tp

ROWS, D = 5, 12
F32 = 4
FAR = [0x10000 * i for i in range(1, 40)]
CONFIG = tp.Norm(ROWS, D, 3, tp.TP_F32, 1e-6, FAR[30], FAR[31], FAR[32])
FORWARD = ("x", "y", "z", "x_out", "n")
BACKWARD = ("x", "y", "z", "dx_out", "dn", "dx", "dy", "dz")


def call(names, at, dw=None, work=FAR[35], nb=1 << 30):
    m = [C.byref(tp.Matrix(*at.get(k, (FAR[i], D)))) for i, k in enumerate(names)]
    if names is FORWARD:
        return tp.load().tp_norm_forward(C.byref(CONFIG), *m, None)
    dw = dw or (FAR[20], FAR[21], FAR[22])
    return tp.load().tp_norm_backward(C.byref(CONFIG), *m, *dw, work, nb, None)


def refused(rc, *names):
    assert rc == tp.TP_EINVAL and "overlaps" in tp.last_error(), (rc, tp.last_error())
    assert all(n in tp.last_error() for n in names), tp.last_error()


@pytest.mark.parametrize("shift,ld", [(4, D), (-4, D), (D * 4, D), (4, 3 * D), (3 * D * F32 + 44, 3 * D),
                                      (-3 * D * F32 - 4, 3 * D), (-3 * D * F32 * 4 - 44, 3 * D)])
@pytest.mark.parametrize("names,out,other", [
    (FORWARD, "x_out", "x"), (FORWARD, "n", "z"), (FORWARD, "x_out", "n"), (BACKWARD, "dx", "dn"),
    (BACKWARD, "dy", "y"), (BACKWARD, "dz", "dx"), (BACKWARD, "dy", "dz"), (BACKWARD, "dz", "x")])
def test_rows_that_share_some(names, out, other, shift, ld):
    refused(call(names, {out: (0x900000 + shift, ld), other: (0x900000, ld)}), out, other)


def test_outputs_that_are_one_buffer():
    refused(call(FORWARD, {"x_out": (FAR[3], D), "n": (FAR[3], D)}), "x_out", "n")
    refused(call(BACKWARD, {"dx": (FAR[3], D), "dz": (FAR[3], D)}), "dx", "dz")
    refused(call(BACKWARD, {}, dw=(FAR[20], FAR[20] + 4 * (D - 1), FAR[22])), "dw_post", "dscale")


def test_unlike_pitches():
    refused(call(FORWARD, {"n": (0x900000, 2 * D), "y": (0x900000, D)}), "n", "y")
    refused(call(FORWARD, {"n": (0x900000 + 4 * D, D), "y": (0x900000, 2 * D)}), "n", "y")


def test_weights_and_the_workspace():
    refused(call(FORWARD, {"n": (FAR[32] - 4, D)}), "n", "w_pre")
    refused(call(BACKWARD, {"dy": (FAR[31] - 4 * (ROWS * D - 1), D)}), "dy", "scale")
    refused(call(BACKWARD, {"dx": (FAR[35] + 256, D)}), "dx", "the workspace")
    refused(call(BACKWARD, {"dn": (FAR[35] + 256, D)}), "the workspace", "dn")
    refused(call(BACKWARD, {}, dw=(FAR[0] + 8, FAR[21], FAR[22])), "dw_post", "x")
