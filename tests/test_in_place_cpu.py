"""Host-only: kernels that may be told to write where they read (layer norm with y in x's place, its gradient with dx in x's or dy's place, dropout) give
the compiler no word that they do not."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1810_09868_amd", "csrc")


def parameters(source, kernel):
    """{name: type} of a kernel's parameters."""
    text = re.search(r"\b%s\(([^)]*)\)" % kernel, source).group(1)
    return {p.split("*")[-1].replace("__restrict__", "").split()[-1]: p for p in text.split(",")}


@pytest.mark.parametrize("kernel,places", [("layer_norm_kernel", ("x", "y")), ("layer_norm_long_kernel", ("x", "y")), ("layer_norm_bwd_kernel", ("x", "dy", "dx")),
                                           ("layer_norm_bwd_long_kernel", ("x", "dy", "dx")), ("dropout_kernel", ("x", "y"))])
def test_what_may_be_the_same_place_is_not_said_to_be_apart(kernel, places):
    with open(os.path.join(CSRC, "norm.hip")) as f:
        found = parameters(f.read(), kernel)
    for name in places:
        assert "*" in found[name] and "__restrict__" not in found[name], (kernel, found[name])
