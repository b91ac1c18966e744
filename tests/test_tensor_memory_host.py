"""CPU test: no kernel of this library waits for tensor memory (csrc/tcgen05.h says why none may)."""

import os
import re

import paper_2006_03108_b200

CSRC = os.path.join(os.path.dirname(paper_2006_03108_b200.__file__), "csrc")


def test_every_kernel_with_tensor_memory_states_that_its_blocks_fit():
    """A kernel that allocates columns has a static_assert of its sizes, which the build checks, and takes no shared memory beside what it states there.
    The statement itself holds for blocks of any sizes that pass it."""
    kernels = {}
    for name in sorted(os.listdir(CSRC)):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
        stated = set(re.findall(r'static_assert\([^;]*tensor_blocks_fit[^;]*?(\w+)"\);', text))
        stated |= set(re.findall(r'static_assert\([^;]*"tensor_blocks_fit: (\w+)"\);', text))
        for m in re.finditer(r"__global__ void __launch_bounds__\((?:[^()]|\([^()]*\))*\)\s*(\w+)\(", text):
            brace = text.index("{", m.end())
            depth, end = 1, brace + 1
            while depth:
                depth += {"{": 1, "}": -1}.get(text[end], 0)
                end += 1
            body = text[brace:end]
            if "tcgen05.alloc" in body:
                kernels[m.group(1)] = m.group(1) in stated
                assert not re.search(r"(?<!extern )__shared__", body), m.group(1)
    assert {"affine_kernel_pair", "affine_kernel_split", "affine_kernel_quad", "affine_dw_kernel", "affine_fp8_pair_kernel", "affine_fp8_few_kernel"} <= set(kernels)
    assert all(kernels.values()), [k for k, v in kernels.items() if not v]
    sm, block, least = 228, 1, 80                                    # KB; as in tcgen05.h
    header = open(os.path.join(CSRC, "tcgen05.h")).read()
    assert "kSmSharedBytes = %d * 1024" % sm in header and "kTensorSharedBytes = %d * 1024" % least in header
    fits = [(s, c) for s in range(least, sm) for c in (32, 64, 128, 256, 512) if c <= 256 or s + least + 2 * block > sm]
    for s, c in fits:
        for s2, c2 in fits:
            assert s + s2 + 2 * block > sm or c + c2 <= 512
    assert 3 * (least + block) > sm
