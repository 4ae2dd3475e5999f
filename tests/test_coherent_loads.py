"""Kernels that are launched before the kernel in front of them has ended (programmatic dependent launch: they open with pdl_enter) use no
non-coherent loads, which are only valid for memory that is constant while a kernel runs: no __ldg in them or in the functions that they
call, and no input pointer of theirs that is __restrict__, through which the compiler may load in the same way."""
from __future__ import annotations

import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_07114_b200", "csrc")


def _functions():
    """(file, name, signature, body) of every __global__ or __device__ function of the headers and of the files with such kernels."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh"))):
        src = re.sub(r"//[^\n]*", "", open(path).read())
        if path.endswith(".cu") and "pdl_enter()" not in src:
            continue
        for m in re.finditer(r"__(?:global|device)__", src):
            brace, semi = src.find("{", m.end()), src.find(";", m.end())
            if brace < 0 or (0 <= semi < brace):
                continue                                                   # a variable
            depth, end = 0, brace
            while True:
                depth += (src[end] == "{") - (src[end] == "}")
                end += 1
                if depth == 0:
                    break
            signature = src[m.start():brace]
            name = re.findall(r"(\w+)\s*\(", re.sub(r"__launch_bounds__\([^)]*\)", "", signature))
            yield os.path.basename(path), name[0] if name else "", signature, src[brace:end]


def test_no_non_coherent_loads_where_a_kernel_starts_early():
    early = 0
    for file, name, signature, body in _functions():
        plain_kernel = "__global__" in signature and "pdl_enter()" not in body
        early += "__global__" in signature and not plain_kernel
        if plain_kernel:
            continue
        assert "__ldg(" not in body, f"{file}: {name} uses __ldg"
        assert not re.search(r"const [\w ]+\*\s*__restrict__", signature), f"{file}: {name} has an input pointer that is __restrict__"
    assert early >= 20
