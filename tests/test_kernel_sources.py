"""What the sources of kernels that start under the kernel before them may not say."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2101_10761_b200", "csrc")


def kernels(name):
    """(name, parameters, first half of the body) of the kernels of a file."""
    text = open(os.path.join(CSRC, name)).read()
    for m in re.finditer(r"__global__ void[^;{]*?\b(\w+_kernel)\((.*?)\)\s*\{", text, re.S):
        yield m.group(1), m.group(2), text[m.end():m.end() + 4000].split("\n}\n")[0]


# Inputs that no kernel of their call writes, read behind a kernel of the call that is not started early itself.
UNCHANGED = {("momentum_kernel", "grad"), ("again_kernel", "grad")}


@pytest.mark.parametrize("name", ["sidco_embedding.cu", "sidco_dropout.cu", "sidco_cross_entropy.cu", "sidco_mx4.cu",
                                  "sidco_mx4_matmul.cu", "sidco_orthogonalize.cu"])
def test_kernels_that_start_early_claim_no_input_as_unchanging(name):
    """They are resident while the kernel before them still writes what they are going to read: const __restrict__, which says
    that nothing changes it as long as they run, would allow reads ahead of the wait and past the coherent caches."""
    seen = 0
    for kernel, parameters, body in kernels(name):
        if not re.search(r"\b(wait_prerequisites|begin)\(\);", body):
            continue
        seen += 1
        claimed = [p.split()[-1] for p in parameters.split(",") if re.match(r"\s*const\b", p) and "__restrict__" in p]
        claimed = [p for p in claimed if (kernel, p) not in UNCHANGED]
        assert not claimed, (kernel, claimed)
        assert "__ldg(" not in body, kernel
    assert seen >= 2
