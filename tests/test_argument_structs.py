"""The packed arguments of the binding against the structures of include/hif4.h.  No GPU."""
import os
import re
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODES = {"int64_t": "q", "int": "i", "float": "f"}


def fields(name):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hif4.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^{}]*)\} " + name + ";", text).group(1)
    out = []
    for decl in filter(None, (d.strip() for d in body.split(";"))):
        kind, names = re.match(r"(?:const )?(\w+)(.*)", decl, flags=re.S).groups()
        for n in names.split(","):
            out.append((n.replace("*", "").strip(), "P" if "*" in n else CODES.get(kind, "i")))      # enumerations are ints
    return out


@pytest.mark.parametrize("name", ["hif4_block_norm_args", "hif4_block_norm_backward_args", "hif4_linear_act_args", "hif4_linear_act_backward_args"])
def test_format_follows_the_fields(name):
    import paper_2602_11287_b200.binding as b
    assert b.ARGUMENT_FORMATS[name] == "".join(code for _, code in fields(name)) + "0q"


def test_sizes_and_offsets_are_those_of_the_c_compiler(tmp_path):
    import paper_2602_11287_b200.binding as b
    lines = []
    for name in b.ARGUMENT_FORMATS:
        lines.append(f'printf("{name} %zu", sizeof({name}));')
        lines += [f'printf(" %zu", offsetof({name}, {f}));' for f, _ in fields(name)]
        lines.append('printf("\\n");')
    src = tmp_path / "offsets.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"hif4.h\"\nint main(void) {" + "\n".join(lines) + "return 0; }\n")
    exe = tmp_path / "offsets"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines():
        name, size, *offsets = line.split()
        fmt = b.ARGUMENT_FORMATS[name]
        codes = fmt[:-2]
        assert struct.calcsize(fmt) == int(size)
        assert [struct.calcsize(codes[:i + 1]) - struct.calcsize(codes[i]) for i in range(len(codes))] == [int(o) for o in offsets]


def test_the_header_is_plain_c(tmp_path):
    src = tmp_path / "h.c"
    src.write_text('#include "hif4.h"\nint main(void) { return 0; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o", str(tmp_path / "h.o")], check=True)
