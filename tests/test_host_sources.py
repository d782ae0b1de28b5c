"""What the kernels' sources must not hold."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_13519_b200", "csrc")


def _sources():
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            yield name, f.read()


@pytest.mark.parametrize("word", ["cta_group::2", ".multicast::cluster"])
def test_no_kernel_of_cta_pairs(word):
    """Tensor memory allocated by a pair of CTAs (cta_group::2) has been seen to stand still for good, with a cause that is not known, and
    the allocation has no bounded form: no kernel may have one."""
    assert [name for name, text in _sources() if re.search(re.escape(word), text)] == []


def test_no_load_for_constant_data_in_kernels_that_start_early():
    """A kernel launched under programmatic dependent launch runs before the data of the kernel ahead of it are there; ld.global.nc (__ldg)
    is for data that nobody writes while the kernel runs, and the dependency wait does not order it.  Only the kernel that reads codes and
    scales back has such loads, and it is launched without the attribute."""
    for name, text in _sources():
        if name == "mxfp4.cu":
            first = text.index("mx_dequantise_kernel(")
            text = text[:first] + text[text.index("__global__", first):]
            assert re.search(r"mx_dequantise_kernel<T, V><<<", text)
        assert not re.search(r"__ldg\(|ld\.global(\.\w+)*\.nc|__restrict__", text), name
