"""Indices of the built library's kernels stay whole numbers (CPU).

HIP's max and min of a signed and an unsigned number are those of 64-bit floats: -1 that an
unsigned count has wrapped to 2^32 - 1 then stays that large, and the index it becomes lies
gigabytes past its array.  No kernel here has any other use for the larger or smaller of two
64-bit floats, or makes whole numbers of them, so the machine code holds none of these
instructions."""
from __future__ import annotations

import os
import re
import subprocess

import pytest

from test_matrix_waits import OBJDUMP

FLOATS = re.compile(r"^\t(v_(?:max|min)_f64\S*|v_cvt_[iu]32_f64\S*)", re.M)


def found(text):
    """(kernel, instruction) of each such instruction."""
    out = []
    for part in re.split(r"^(?=[0-9a-f]+ <)", text, flags=re.M):
        m = re.match(r"[0-9a-f]+ <(.+)>:", part)
        out += [(m.group(1), x) for x in FLOATS.findall(part)] if m else []
    return out


def test_the_search_sees_them():
    code = ("0000000000001000 <kernel>:\n\tv_cvt_f64_u32_e32 v[4:5], s4  // 000000001000: 00\n"
            "\tv_max_f64 v[4:5], v[4:5], 0  // 000000001008: 00\n"
            "\tv_cvt_i32_f64_e32 v3, v[4:5]  // 000000001010: 00\n")
    assert found(code) == [("kernel", "v_max_f64"), ("kernel", "v_cvt_i32_f64_e32")]


def test_no_index_goes_through_floats(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no disassembler")
    from paper_1505_02890_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_1505_02890_amd.build import build
        build()
    lib = tmp_path / "lib.so"
    lib.write_bytes(open(_lib.LIB_PATH, "rb").read())
    subprocess.run([OBJDUMP, "--offloading", str(lib)], cwd=tmp_path, check=True,
                   capture_output=True)
    parts = sorted(p for p in tmp_path.iterdir() if "gfx950" in p.name)
    assert parts
    for p in parts:
        text = subprocess.run([OBJDUMP, "-d", str(p)], check=True, capture_output=True,
                              text=True).stdout
        assert "s_endpgm" in text
        assert found(text) == [], p.name
