"""The cache's argument struct as a C compiler lays it out, against the binding's."""
import ctypes
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_cache_struct_of_the_binding_matches_the_header(tmp_path):
    from paper_2602_17698_b200.binding import Kv8CacheStruct
    names = [f for f, _ in Kv8CacheStruct._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "scalebits.h"\nint main(void) {\n  printf("%zu", sizeof(sb_kv8_cache));\n' +
                   "".join(f'  printf(" %zu", offsetof(sb_kv8_cache, {f}));\n' for f in names) + "  return 0;\n}\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got[0] == ctypes.sizeof(Kv8CacheStruct)
    assert got[1:] == [getattr(Kv8CacheStruct, f).offset for f in names]
