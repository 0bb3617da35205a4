"""The public headers are C, and the library exports what they declare. No GPU."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2606_14598_b200 import binding

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
HEADERS = sorted(h for h in os.listdir(INCLUDE) if h.endswith(".h"))


@pytest.mark.parametrize("header", HEADERS)
def test_header_is_c(header):
    source = f'#include "{header}"\nint main(void) {{ return 0; }}\n'
    r = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-fsyntax-only", "-I", INCLUDE, "-x", "c", "-"], input=source, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


@pytest.mark.parametrize("header", HEADERS)
def test_library_exports_what_the_header_declares(header):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(INCLUDE, header)).read(), flags=re.S)
    names = set(re.findall(r"\b((?:int8|mxfp4|kv_cache)_[a-z0-9_]+)\s*\(", text))
    assert names
    lib = ctypes.CDLL(binding.LIB_PATH)
    assert not [n for n in names if not hasattr(lib, n)]
