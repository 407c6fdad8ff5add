"""include/kvio_attn.h without a GPU: the library exports what it declares, the binding's constants and structs are its."""
import ctypes
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TEXT = open(os.path.join(ROOT, "include", "kvio_attn.h")).read()


def test_library_exports_every_declared_symbol():
    import paper_2508_18572_amd as kv
    names = sorted(set(re.findall(r"^kvio_status (kvio_[a-z_]+)\(", TEXT, flags=re.M)))
    assert names == ["kvio_append", "kvio_attend", "kvio_attend_workspace"]
    lib = ctypes.CDLL(kv.LIB_PATH)
    assert all(hasattr(lib, n) and hasattr(kv, n) for n in names)


def test_python_constants_match_the_header():
    import paper_2508_18572_amd.attn as A
    consts = dict(re.findall(r"#define (KVIO_[A-Z0-9_]+) (0x[0-9a-fA-F]+|\d+)\b", TEXT))
    assert len(consts) == 4
    for name, value in consts.items():
        assert getattr(A, name) == int(value, 0), name


def test_ctypes_structs_match_the_c_layout(tmp_path):
    import paper_2508_18572_amd.attn as A
    structs = ("kvio_batch", "kvio_append_args", "kvio_attend_args")
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "kvio_attn.h"', "int main(void) {"]
    for st in structs:
        lines.append(f'    printf("{st} size %zu\\n", sizeof({st}));')
        lines += [f'    printf("{st} {f} %zu\\n", offsetof({st}, {f}));' for f, _ in getattr(A, st)._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["    return 0;", "}"]) + "\n")
    exe = str(tmp_path / "layout")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split("\n")
    c = {(a, b): int(v) for a, b, v in (ln.split() for ln in out if ln)}
    for st in structs:
        cls = getattr(A, st)
        assert ctypes.sizeof(cls) == c[(st, "size")], st
        for f, _ in cls._fields_:
            assert getattr(cls, f).offset == c[(st, f)], (st, f)
