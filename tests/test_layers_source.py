"""Rules of the layers' kernels that no run can show to be broken, checked in their source: a warp-wide .aligned instruction is
reached by a converged warp."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2305_12213_b200", "csrc")


def functions(name):
    """(name, body) of every function of a source file, comments taken out."""
    text = open(os.path.join(CSRC, name)).read()
    text = re.sub(r"//[^\n]*", "", text)
    out = []
    for m in re.finditer(r"(?:__device__|__global__)[^;{}]*?(\w+)\((?:[^()]|\([^()]*\))*\)\s*\{", text):
        depth, i = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[i], 0)           # those in assembly strings are balanced too
            i += 1
        out.append((m.group(1), text[m.end():i - 1]))
    return out


def instructions(body):
    """Places of warp-wide aligned instructions: inline assembly, and calls of the wrappers that leave convergence to callers."""
    return [m.start() for m in re.finditer(r"asm volatile\(\s*\"[^;]*?\.aligned|tc::tmem_(?:load32|alloc|dealloc)\(", body)]


@pytest.mark.parametrize("name,at_least", [("layer_gemm.cuh", 7), ("embedding.cu", 1)])
def test_aligned_instructions_are_reached_by_converged_warps(name, at_least):
    found = 0
    for function, body in functions(name):
        for at in instructions(body):
            before = body.find("__syncwarp();")
            assert 0 <= before < at, f"{function}: an aligned instruction without __syncwarp() before it"
            # a wrapper: nothing but the choice of the form lies between
            assert len(re.findall(r"\bfor\b|\bwhile\b", body[before:at])) == 0, function
            found += 1
    assert found >= at_least
