"""The two ways in which the binding writes a qift_linear_output agree with one another and with the header (CPU)."""
import ctypes
import os
import re
import subprocess

from paper_2606_02823_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_both_layouts_are_the_same_bytes():
    a, b = (11, 22, 33, 44, 55, 66), (1 << 63, 2 << 40, 3, 4 << 33, 2 ** 31 - 1, 6)
    pair = (binding.LinearOutput * 2)(binding.LinearOutput(*a), binding.LinearOutput(*b))
    assert binding._GATE_UP.pack(*a, *b) == bytes(pair)


def test_the_header_has_that_layout(tmp_path):
    fields = [f for f, _ in binding.LinearOutput._fields_]
    source = tmp_path / "layout.c"
    offsets = ", ".join(f"(int)offsetof(qift_linear_output, {f})" for f in fields)
    source.write_text('#include "qift.h"\n#include <stdio.h>\nint main(void) { int v[] = {(int)sizeof(qift_linear_output), %s}; '
                      'for (int i = 0; i < %d; ++i) printf("%%d ", v[i]); return 0; }\n' % (offsets, len(fields) + 1))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(source), "-o", str(tmp_path / "layout")], check=True)
    got = [int(x) for x in re.findall(r"\d+", subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout)]
    assert got == [ctypes.sizeof(binding.LinearOutput)] + [getattr(binding.LinearOutput, f).offset for f in fields]
