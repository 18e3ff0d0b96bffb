"""Kernels that allocate TMEM let the next kernel of the stream start only behind the barrier after the allocation: a CTA of
that kernel on the same SM could otherwise hold the columns, waiting for this grid to end, while this CTA waits for them."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2502_19864_gb300", "csrc")


def kernels():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        source = re.sub(r"//[^\n]*", "", open(path).read())
        for body in source.split("__global__")[1:]:
            if "tcgen05.alloc" in body:
                yield pytest.param(body, id=os.path.basename(path) + ":" + re.search(r"(\w+_kernel)\b", body).group(1))


@pytest.mark.parametrize("body", list(kernels()))
def test_dependents_start_behind_the_allocation(body):
    allocated = body.rindex("tcgen05.alloc")
    barrier = body.index("__syncthreads()", allocated)
    assert body.index("pdl_trigger()") > barrier
