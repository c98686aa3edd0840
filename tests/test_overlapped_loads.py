"""What a kernel reads of the launch before it, which may still be running when it starts, is never loaded as a constant: CUDA allows such loads (``__ldg``, or
what a compiler makes of a pointer to const that is ``__restrict__``) only of memory that nobody writes as long as the kernel lives."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_17644_b200", "csrc")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


@pytest.mark.parametrize("file,kernel,pointers", [
    ("attn_decode_sm100.cuh", "decode_project_kernel", ("part_o", "part_ml")),
    ("attn_decode8_sm100.cuh", "decode8_join_kernel", ("part_o", "part_ml")),
    ("attn_bwd_sm100.cuh", "bwd_dkpe_reduce_kernel", ("dk_rope",)),
    ("attn_bwd_sm100.cuh", "bwd_dkpe_convert_kernel", ("dkpe_acc",)),
    ("attn_bwd_fused_sm100.cuh", "bwd_dq_convert_kernel", ("dq_acc",)),
    ("rope_sm100.cuh", "latent_norm_sums_kernel", ("partial",)),
])
def test_arguments(file, kernel, pointers):
    text = source(file)
    found = re.search(rf"^{kernel}\((.*?)\)\s*\{{", text, re.S | re.M)
    assert found, kernel
    for name in pointers:
        [declared] = [a for a in found[1].split(",") if re.search(rf"\b{name}$", a.strip())]
        assert not ("const" in declared and "__restrict__" in declared), declared
        assert not re.search(rf"__ldg\([^;]*\b{name}\b", text), name


@pytest.mark.parametrize("name", ["q_scale", "part_o", "part_ml"])
def test_members(name):
    for file in ("attn_decode8_sm100.cuh", "attn_decode_sm100.cuh"):
        assert not re.search(rf"__ldg\([^;]*\.{name}\b", source(file)), (file, name)
