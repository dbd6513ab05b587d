"""Rules that the CUDA sources keep and that no run can show to be kept: what breaks them goes right until the timing changes."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2508_18182_b200", "csrc")


def _source(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def _kernels(text):
    """(name, body) of every kernel of a source."""
    for m in re.finditer(r"__global__\s+void\s*(?:__launch_bounds__\((?:[^()]|\([^()]*\))*\))?\s*(\w+)\s*\(", text):
        start = text.index("{", m.end())
        depth, i = 1, start + 1
        while depth:
            depth += {"{": 1, "}": -1}.get(text[i], 0)
            i += 1
        yield m.group(1), text[start:i]


CUDA_SOURCES = sorted(f for f in os.listdir(CSRC) if f.endswith(".cu"))


def test_kernels_are_found():
    names = {k for f in CUDA_SOURCES for k, _ in _kernels(_source(f))}
    assert {"rmsnorm_gain_kernel", "blockscale_pair_kernel", "add_rmsnorm_kernel", "rope_kernel"} <= names and len(names) > 20


def test_no_block_reaches_into_another_one_that_may_not_have_started():
    """Shared memory of another block of the cluster may be accessed only after a barrier of the cluster."""
    reaching = 0
    for f in CUDA_SOURCES:
        for name, body in _kernels(_source(f)):
            first = re.search(r"\bmap_to_cta\s*\(", body)
            if not first:
                continue
            reaching += 1
            # a lambda or a function before the barrier that only names an address counts as an access: none does
            assert re.search(r"\bcluster_(sync_all|all_started)\s*\(", body[:first.start()]), (f, name)
            if "cluster_all_started" in body:
                assert body.index("cluster_started") < body.index("cluster_all_started"), (f, name)
    assert reaching >= 3


def test_kernels_launched_early_read_nothing_through_the_non_coherent_path():
    """A kernel that starts while the one before it drains may not use loads for data that is constant while it runs."""
    early = [f for f in CUDA_SOURCES if re.search(r"\blaunch_early\s*\(", _source(f))]
    assert {"block_kernels.cu", "blockscale_gemm.cu"} <= set(early)
    for f in early + ["ptx.cuh", "common.cuh"]:
        assert not re.search(r"__ldg\b|ld\.global(\.\w+)*\.nc|__restrict__", _source(f)), f
    for f in early:
        for name, body in _kernels(_source(f)):
            assert re.search(r"\bafter_predecessor\s*\(\s*\)", body), (f, name)


def test_scale_warps_that_give_up_wait_for_their_copies():
    """A warp that leaves after a wait ran out may not leave asynchronous copies into shared memory behind."""
    text = _source("blockscale_gemm.cu")
    body = text[text.index("if (!walk.more() || !fetch(0)) return;"):]
    body = body[:body.index("__global__")]
    leave = body[body.index("!fetch(i ^ 1)"):]
    assert re.match(r"!fetch\(i \^ 1\)\)\s*\{\s*asm volatile\(\"cp\.async\.wait_all;\"[^;]*\);\s*return;", leave), leave[:200]
