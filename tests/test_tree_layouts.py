"""The tables' descriptor as the C compiler sees the header and as the binding fills it (no GPU)."""
import ctypes
import os
import subprocess

from paper_2503_01586_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_tables_descriptor(tmp_path):
    names = [f[0] for f in binding.TablesDesc._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "elitekv.h"\nint main(void){printf("%zu\\n", sizeof(elitekv_tables));' +
                   "".join(f'printf("%zu\\n", offsetof(elitekv_tables, {n}));' for n in names) + "return 0;}")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(binding.TablesDesc)] + [getattr(binding.TablesDesc, n).offset for n in names]
