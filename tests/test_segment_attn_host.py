"""Cross and shared-prefix attention at the C boundary, without a GPU: the binding's argument structures have the header's
layout, and calls without a context or arguments are refused."""
import ctypes
import os
import subprocess

import pytest

from paper_2609_38984_b200 import build as swam_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    swam_build.build_library()
    from paper_2609_38984_b200 import swam
    return swam.load_library()


@pytest.mark.parametrize("c_name,py_name", [("swam_cross_args", "SwamCrossArgs"), ("swam_prefix_args", "SwamPrefixArgs")])
def test_argument_structures_match_the_header(tmp_path, c_name, py_name):
    from paper_2609_38984_b200 import swam
    cls = getattr(swam, py_name)
    fields = [f for f, _ in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "swam.h"\nint main(void) {\n'
                   + "".join(f'  printf("%zu %zu\\n", offsetof({c_name}, {f}), sizeof((({c_name}*)0)->{f}));\n' for f in fields)
                   + f'  printf("%zu 0\\n", sizeof({c_name}));\n  return 0;\n}}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    lines = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")
    for f, line in zip(fields, lines):
        assert tuple(map(int, line.split())) == (getattr(cls, f).offset, getattr(cls, f).size), f
    assert int(lines[len(fields)].split()[0]) == ctypes.sizeof(cls)


@pytest.mark.parametrize("name,py_name", [("swam_cross_attn", "SwamCrossArgs"), ("swam_prefix_attn", "SwamPrefixArgs")])
def test_calls_without_a_context_are_refused(lib, name, py_name):
    from paper_2609_38984_b200 import swam
    args, bytes_ = getattr(swam, py_name)(), ctypes.c_size_t(7)
    assert getattr(lib, name)(None, ctypes.byref(args), None) == swam.ERR_INVALID_ARG
    assert getattr(lib, name)(None, None, None) == swam.ERR_INVALID_ARG
    assert getattr(lib, name + "_scratch_bytes")(None, ctypes.byref(args), ctypes.byref(bytes_)) == swam.ERR_INVALID_ARG
    assert bytes_.value == 7
