"""Rules of the layers' kernels that no run can show to be broken, checked in their source: a warp-wide .aligned instruction is
reached by a converged warp, and a wait's verdict is the same in all lanes of a warp that goes on as one."""
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


def test_waits_have_one_verdict_for_a_warp():
    """A time-limited wait ends in each lane on its own: its result is shared by the warp before anything branches on it."""
    waits = 0
    for function, body in functions("layer_gemm.cuh"):
        for line in body.splitlines():
            if "tc::mbar_wait(" in line:
                shared = "__all_sync(0xFFFFFFFFu, tc::mbar_wait(" in line
                one_lane = "if (lane == 0) ready = tc::mbar_wait(" in line and "__shfl_sync(0xFFFFFFFFu, ready, 0)" in body
                assert shared or one_lane, (function, line.strip())
            waits += line.count("mbar_wait(") + line.count("warp_wait(")
    assert waits >= 6


def test_giving_up_leaves_no_arrival_for_the_other_cta():
    """Every barrier that the products arrive on in both CTAs of a pair is waited for in both; the one that only the CTA that gives
    up waits for is arrived on there alone."""
    body = dict(functions("layer_gemm.cuh"))["layer_gemm_kernel"]
    both = re.findall(r"mma_commit<CG>\(&(\w+)", body)
    assert sorted(both) == ["empty_bar", "ready_bar"]
    waited = re.findall(r"(?:warp_wait|tc::mbar_wait)\(&(\w+)", body)
    assert all(waited.count(b) >= 1 for b in both)
    assert re.findall(r"mma_commit_here<CG>\(&(\w+)", body) == ["drain_bar"]
    here = dict(functions("layer_gemm.cuh"))["mma_commit_here"]
    assert "multicast" not in here and "cta_group::2" in here
