"""The header is plain C99, and describes the same structures in C99, C11 and C++."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = """
#include <stddef.h>
#include <stdio.h>
#include "luvc.h"
int main(void) {
    luvc_kv_cache c;
    float scale = 1.0f;
    c.k_scale = &scale;
    c.v_scale = &scale;
    printf("%d %d %d %d %d", (int)sizeof c, (int)offsetof(luvc_kv_cache, k_scale), (int)offsetof(luvc_kv_cache, v_scale),
           (int)offsetof(luvc_kv_cache, layers), c.k_scale == c.v_scale);
    return 0;
}
"""


@pytest.mark.parametrize("compiler,standard,suffix", [("gcc", "c99", ".c"), ("gcc", "c11", ".c"), ("gcc", "gnu99", ".c"), ("g++", "c++11", ".cpp")])
def test_the_header_compiles(tmp_path, compiler, standard, suffix):
    assert shutil.which(compiler)
    source, program = tmp_path / ("header" + suffix), tmp_path / "header"
    source.write_text(SOURCE)
    subprocess.run([compiler, "-std=" + standard, "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(source), "-o", str(program)],
                   check=True, capture_output=True)
    import paper_2512_09010_b200 as luvc
    s = luvc.KvCacheStruct
    import ctypes
    want = [ctypes.sizeof(s), s.k_scale.offset, s.v_scale.offset, s.layers.offset, 1]
    assert subprocess.run([str(program)], check=True, capture_output=True, text=True).stdout.split() == [str(x) for x in want]
