"""Calls whose output may lie in an input's memory: the kernels promise the compiler nothing else, and in place gives the bits that another buffer gets."""
import os
import re

import pytest
import torch

from paper_2412_07752_amd import api

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2412_07752_amd", "csrc")

# outputs that the header allows to be one of these inputs, by the names that the kernels give them
MAY_BE = {"flashrnn_norm.hip": {"y": ["x"], "dx": ["dy", "x"]}, "flashrnn_loss.hip": {"dlogits": ["logits"]}, "flashrnn_clip.hip": {"out": ["in"]}}


@pytest.mark.parametrize("name", sorted(MAY_BE))
def test_pointers_that_may_be_the_same_are_not_restricted(name):
    """A kernel that writes through one of two such pointers must not call either __restrict__."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    seen = 0
    for head in re.findall(r"__global__[^{;]*?\)\s*void (\w+\([^{;]*\))\s*\{", text) + re.findall(r"struct (?:Problem|Table) \{.*?\};", text, re.S):
        pointers = {}
        for a in re.split(r"[,;({}]", head):   # parameters, or members (a list of them shares what stands before the first)
            if m := re.search(r"(\w+)(?:\[\w+\])?\)?\s*$", a):
                pointers[m.group(1)] = a
        for out, inputs in MAY_BE[name].items():
            if out in pointers and "const" not in pointers[out]:
                seen += 1
                for a in [out] + inputs:
                    assert "__restrict__" not in pointers.get(a, ""), (head.split("(")[0].split()[0], pointers[a].strip())
    assert seen, "no kernel or descriptor with such an output"


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width", [(1, 8), (40, 5), (40, 100), (513, 1111), (40, 3000), (70_001, 768), (2_500, 12_001), (5, 30_000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layer_norm_in_place(rows, width, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x, w, b = (torch.randn(s, generator=gen, device="cuda") for s in ((rows, width), (width,), (width,)))
    x = x.to(dtype)
    want = api.flashrnn_layer_norm_fwd(x, w, b)
    got = api.flashrnn_layer_norm_fwd(x, w, b, y=x)
    assert got[0] is x and all(torch.equal(p, q) for p, q in zip(got, want))
