"""Rules that the sources of overlapped launches keep (host only).

launch_overlapped lets a kernel be resident before the kernel ahead of it on the stream has ended.  Its
inputs may still be written then, so they are not constant during its life, and must not be declared in
the form that allows the compiler to read them through the non-coherent path; and every such kernel calls
wait_for_previous().
"""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_07713_gb300", "csrc")


def sources():
    out = {}
    for name in sorted(os.listdir(CSRC)):
        if name.endswith(".cu"):
            with open(os.path.join(CSRC, name)) as f:
                text = re.sub(r"//[^\n]*", "", f.read())
            if "launch_overlapped(" in text:
                out[name] = text
    return out


def kernels(text):
    """name: (parameters, body) of every __global__ function."""
    out = {}
    for m in re.finditer(r"__global__\s+void\s+(?:__launch_bounds__\(.*?\)\s*\n)?\s*(\w+)\(", text):
        depth, i = 1, m.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[i], 0)
            i += 1
        start = text.index("{", i)
        depth, j = 1, start + 1
        while depth:
            depth += {"{": 1, "}": -1}.get(text[j], 0)
            j += 1
        out[m.group(1)] = (text[m.end():i - 1], text[start:j])
    return out


@pytest.mark.parametrize("name", sorted(sources()))
def test_inputs_of_overlapped_kernels_are_not_declared_constant(name):
    found = kernels(sources()[name])
    assert found
    for kernel, (parameters, body) in found.items():
        constant = [p.strip() for p in parameters.split(",") if re.search(r"\bconst\b[^,]*\*\s*__restrict__", p)]
        assert not constant, (kernel, constant)
        assert "__ldg(" not in body and "ld.global.nc" not in body, kernel


@pytest.mark.parametrize("name", sorted(sources()))
def test_overlapped_kernels_wait_for_the_one_before(name):
    for kernel, (_, body) in kernels(sources()[name]).items():
        assert "wait_for_previous();" in body, kernel
