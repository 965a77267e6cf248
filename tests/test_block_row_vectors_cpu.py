"""Vectors of eight elements anywhere in a row: their loads and stores may assume no more than an element's alignment, since rows
of any length and stride move in them.  What the compiler assumes stands in the device code's loads and stores."""
import re
import subprocess

import pytest

from paper_2002_00104_amd import build

SOURCE = """#include "rows.h"
using namespace pwlq_block;
extern "C" __global__ void store_f32(float *p, const v8f *v) { store8(p, *v); }
extern "C" __global__ void copy_f32(float *p, const float *q) { store8(p, load8(q)); }
extern "C" __global__ void copy_bf16(bf16 *p, const bf16 *q) { store8(p, load8(q)); }
extern "C" __global__ void copy_f16(f16 *p, const f16 *q) { store8(p, load8(q)); }
extern "C" __global__ void copy_i8(int8_t *p, const int8_t *q) { store8(p, load8(q)); }
"""


@pytest.fixture(scope="module")
def functions(tmp_path_factory):
    folder = tmp_path_factory.mktemp("vectors")
    source, out = folder / "vectors.hip", folder / "vectors.ll"
    source.write_text(SOURCE)
    subprocess.run([build.hipcc(), *build.HIPCC_FLAGS, "--cuda-device-only", "-emit-llvm", "-S", "-I" + build.BLOCK, str(source), "-o", str(out)],
                   check=True)
    return dict(re.findall(r"^define [^@]*@(\w+)\(.*?\{(.*?)^\}", out.read_text(), re.M | re.S))


@pytest.mark.parametrize("name,size", [("store_f32", 4), ("copy_f32", 4), ("copy_bf16", 2), ("copy_f16", 2), ("copy_i8", 1)])
def test_vectors_need_an_element_s_alignment(functions, name, size):
    accesses = re.findall(r"(store|load) .*?ptr addrspace\(1\).*?align (\d+)", functions[name])
    assert {kind for kind, _ in accesses} == {"load", "store"}, functions[name]
    for kind, align in accesses:
        if (name, kind) != ("store_f32", "load"):          # its source is a vector of its own
            assert int(align) <= size, (kind, align)
