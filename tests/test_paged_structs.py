"""The ctypes descriptors of the paged calls lie as the header's structs do."""
import ctypes as C
import os
import subprocess

from paper_2402_06082_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = {"subgen_rope": binding.RopeDesc, "subgen_heads": binding.Heads, "subgen_pages": binding.PagesDesc,
           "subgen_batch": binding.BatchDesc, "subgen_qk_args": binding.QkArgs, "subgen_attend_args": binding.AttendArgs}


def test_sizes_and_offsets(tmp_path):
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "subgen.h"', "int main(void) {"]
    want = []
    for name, struct in STRUCTS.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        want.append(C.sizeof(struct))
        for field in struct._fields_:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, field[0]))
            want.append(getattr(struct, field[0]).offset)
    src = tmp_path / "sizes.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    exe = str(tmp_path / "sizes")
    subprocess.check_call(["gcc", "-I" + os.path.join(ROOT, "include"), "-o", exe, str(src)])
    assert [int(x) for x in subprocess.check_output([exe]).split()] == want
