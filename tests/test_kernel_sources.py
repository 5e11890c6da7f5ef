"""Source rules of the kernels' waits and barriers: what no run can show, because it takes a wait that expires in one lane of a warp
only, or a compiler that leaves a warp split."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2009_08065_b200", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def source(path):
    src = open(os.path.join(CSRC, path)).read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", src, flags=re.S))


def closing(src, at, pair="()"):
    depth = 0
    for i in range(at, len(src)):
        depth += (src[i] == pair[0]) - (src[i] == pair[1])
        if depth == 0:
            return i
    raise AssertionError("unbalanced")


# Waits whose answer may differ between the lanes of a warp: each is the argument of a vote, or one thread's alone.
VOTES = r"(?:__all_sync|__syncthreads_and|\w*_all_ok|epilogue_agree)\([^;{}]*$"


@pytest.mark.parametrize("path", [os.path.basename(p) for p in SOURCES])
def test_a_warp_leaves_a_bounded_wait_as_a_whole(path):
    """A lane that gave up alone would leave the others at the next __syncwarp or vote, which then never ends."""
    src = source(path)
    for m in re.finditer(r"\bmbar_wait(?:_suspended)?\(", src):
        before = src[:m.start()]
        line = before[before.rindex("\n") + 1:]
        if re.search(VOTES, line):
            continue
        enclosing = before[max(0, m.start() - 700):]
        one_thread = "lane == 0" in enclosing[enclosing.rfind("if (warp"):].split("{")[0]
        answered = "auto read_ticket = " in enclosing and "epilogue_all_ok(tile != -2)" in src
        assert one_thread or answered, f"{path}: {line.strip()}{src[m.start():m.end() + 40]}"


@pytest.mark.parametrize("path", [os.path.basename(p) for p in SOURCES + glob.glob(os.path.join(CSRC, "*.cuh"))])
def test_cluster_barriers_take_the_whole_warp(path):
    """The aligned forms are undefined for part of a warp: each stands right behind a __syncwarp()."""
    src = source(path)
    for m in re.finditer(r"asm volatile\(\s*\"barrier\.cluster\.", src):
        assert src[:m.start()].rstrip().endswith("__syncwarp();"), f"{path}: {src[m.start():m.end() + 40]}"


def test_tensor_memory_is_read_by_the_whole_warp():
    """The pair kernel's stores go by lanes; what follows them in its loop reads tensor memory and meets at named barriers."""
    src = source("bsp_gemm_fp8.cu")
    at = src.index("{", src.index("void finish_piece("))
    assert src[at:closing(src, at, "{}")].rstrip().endswith("__syncwarp();")
    at = src.index("{", src.index("void epilogue_meet("))
    assert src[at + 1:].lstrip().startswith("__syncwarp();")


@pytest.mark.parametrize("path", [os.path.basename(p) for p in SOURCES if "fp8" in p])
def test_nothing_is_read_ahead_of_the_wait(path):
    """The 8-bit kernels touch global memory only behind the wait for the launch before them, the operands too: which launch that is
    is not theirs to know (another host thread may have put one that rewrites the weight between a quantiser and its product)."""
    src = source(path)
    for m in re.finditer(r"\bif\s*\(([^;{}]*)\)\s*\{?\s*pdl_wait\(\)", src):
        assert re.fullmatch(r"warp [=<>]=? \d+(?: && warp < \d+)?", m.group(1)), f"{path}: a wait that not every call makes: {m.group(0)}"
    assert not re.search(r"\b(?:pdl_wait|begin_work)\([^)]", src), f"{path}: a wait that not every call makes"
    # the kernel that shares a contraction fills its first stages ahead of the CTA's meeting: in each such role the wait comes first
    firsts = list(re.finditer(r"load_[ab]\(i, i\)|scales_[ab]\.load\(P\.[AB], [mn]0, kb0, min", src))
    assert len(firsts) == (4 if "split" in path else 0)
    for m in firsts:
        role = src[:m.start()].rindex("if (warp ==")
        assert "pdl_wait();" in src[role:m.start()], f"{path}: {m.group(0)}"


def kernels(path):
    """name, parameters and body of every kernel of a file, whatever its parameters."""
    src = source(path)
    for m in re.finditer(r"__global__", src):
        name = re.compile(r"(\w+)\s*\((?!\w*Threads|\d|32 \*)").search(src, src.index("\n", m.start()) if "__launch_bounds__" in src[m.start():src.index("\n", m.start())] else m.start())
        end = closing(src, name.end(0) - 1 if src[name.end(0) - 1] == "(" else src.index("(", name.start()))
        body = src.index("{", end)
        yield name.group(1), src[name.end():end], src[body:closing(src, body, "{}") + 1]


def test_every_kernel_of_the_8_bit_files_is_looked_at():
    """The rules of test_launch_overlap.py for the kernels of the 8-bit calls, whose parameters are structures of their own."""
    found = {}
    for path in [os.path.basename(p) for p in SOURCES if "fp8" in p or "adam_batched" in p]:
        for name, params, body in kernels(path):
            found[name] = body
            assert "pdl_wait()" in body and "pdl_launch_dependents()" in body, f"{path}: {name}"
            assert "__ldg(" not in body and not re.search(r"const\s+\w+\s*\*\s*__restrict__", params), f"{path}: {name}"
            assert body.index("pdl_wait()") < body.index("pdl_launch_dependents()"), f"{path}: {name} signals ahead of its wait"
            if "tcgen05.alloc" in body:
                assert body.index("tcgen05.alloc") < body.index("pdl_launch_dependents()"), f"{path}: {name}"
    assert set(found) == {"quantize_kernel", "quantize_both_kernel", "column_sums_kernel", "linear_few_kernel", "product_any_kernel", "gemm_fp8_pair_kernel",
                          "gemm_fp8_split_kernel", "adam_batched_kernel", "adam_stream8_kernel", "adam_batched8_kernel"}
    assert {n for n, body in found.items() if "tcgen05.alloc" in body} == {"gemm_fp8_pair_kernel", "gemm_fp8_split_kernel"}
    for header in glob.glob(os.path.join(CSRC, "*.cuh")):
        assert "__ldg(" not in source(header), header
