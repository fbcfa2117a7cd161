"""An accumulator of the delta rule's kernels takes matrix products of one kind only, by its type: of
unlike kinds, which hipcc puts side by side without a wait, the second has read it too early."""

import os
import subprocess

import pytest

from paper_2111_05188_amd import build

START = """#include "delta.hpp"
using namespace tpk;
__global__ void kernel(floatx4 *p)
{
    typedef Tile<true> TL;
    TL::raw r{};
    const TL::val x = TL::split(p[0]);
"""
ONE_KIND = ["p[0] = TL::mm(r, x, TL::mm(x, r, {p[1]})).v;", "p[0] = TL::mm2(r, r, x, x, TL::mm2(r, r, r, r, {})).v;",
            "p[0] = Tile<false>::mm(p[1], p[2], Tile<false>::mm(p[1], p[1], {p[0]})).v;"]
TWO_KINDS = ["p[0] = TL::mm2(r, r, x, x, TL::mm(r, x, {})).v;", "p[0] = TL::mm(r, x, TL::mm2(r, r, r, r, {})).v;",
             "p[0] = TL::mm(r, x, Tile<false>::mm(p[1], p[2], {})).v;",
             "p[0] = Tile<false>::mm(p[1], p[2], TL::mm2(r, r, x, x, {})).v;",
             "TL::sum2 s; s = TL::mm(r, x, {}); p[0] = s.v;", "floatx4 s = TL::mm(r, x, {}); p[0] = s;"]


def compiles(tmp_path, line):
    src = tmp_path / "kinds.hip"
    src.write_text(START + "    " + line + "\n}\n")
    out = subprocess.run([build.HIPCC, "-x", "hip", *build.FLAGS, "--cuda-device-only", "-fsyntax-only", str(src)],
                         capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 or "error: no " in out.stderr, out.stderr
    return out.returncode == 0


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no hipcc")
def test_products_of_one_kind(tmp_path):
    assert all(compiles(tmp_path, line) for line in ONE_KIND)


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no hipcc")
def test_products_of_two_kinds_do_not_compile(tmp_path):
    assert not any(compiles(tmp_path, line) for line in TWO_KINDS)
