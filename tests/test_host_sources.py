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
