"""The order of wait and release in kernels that are launched as programmatic dependents, read from the sources.

A kernel that reads or writes memory ahead of its own wait (the group FFN kernels, the fused attention block) is only ever the
dependent of the zero-fill, so the zero-fill has to see the work in front of it complete before it releases anyone."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2601_11676_b200", "csrc")
WAIT, RELEASE = "griddepcontrol.wait", "griddepcontrol.launch_dependents"


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def bodies(name):
    """Kernel name -> body, for every __global__ function of a file."""
    text, found = source(name), {}
    for m in re.finditer(r"__global__[^;{]*?(\w+)\s*\((?:[^()]|\([^()]*\))*\)\s*\{", text):
        depth, at = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
        found[m.group(1)] = text[m.end():at]
    return found


def test_the_zero_fill_waits_before_it_releases():
    body = bodies("group_ffn_stream.cu")["zero_partials_kernel"]
    assert 0 <= body.index(WAIT) < body.index(RELEASE) < body.index("make_float4")


def test_token_step_kernels_wait_and_only_the_attention_kernel_releases():
    for name in ("paged_append.cu", "paged_mha.cu", "norm_glue.cu", "mx4_rows.cu", "mx4_product.cu"):
        for kernel, body in bodies(name).items():
            assert "chain_wait()" in body, kernel
            assert (RELEASE in body) == (kernel == "paged_mha_kernel"), kernel


def test_every_release_is_in_a_kernel_that_is_known_for_it():
    known = {"zero_partials_kernel", "group_ffn_stream_kernel", "group_ffn_i4_ring_kernel", "mha_fused_kernel", "paged_mha_kernel"}
    seen = {k for f in sorted(os.listdir(CSRC)) if f.endswith(".cu") for k, body in bodies(f).items() if RELEASE in body}
    assert seen == known
