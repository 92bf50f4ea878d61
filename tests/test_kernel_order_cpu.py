"""Orders in the kernels' sources that the launch chain rests on (fw_internal.h, dep_sync): what no run can show safely."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2010_01546_b200", "csrc")


def kernels():
    """(file and name, body) of every kernel: from its __global__ to the closing brace in the first column."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        with open(path) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        for m in re.finditer(r"^.*__global__", text, re.M):
            body = text[m.start():text.index("\n}", m.start())]
            name = re.search(r"(\w+_kernel)\s*\(", body)
            yield f"{os.path.basename(path)}:{name.group(1) if name else '?'}", body


@pytest.mark.parametrize("name,body", [k for k in kernels() if "tmem_alloc" in k[1]], ids=lambda v: v if ".cu:" in v else "")
def test_tensor_memory_is_taken_after_the_wait(name, body):
    """A grid that the device sets up while its predecessors run holds no tensor memory yet: tcgen05.alloc has no bound, and a
    predecessor that waits for columns this grid holds would never end."""
    waits = [m.start() for m in re.finditer(r"\bdep_(sync|wait)\(\);", body)]
    assert waits and waits[0] < body.index("tmem_alloc"), name


def test_every_kernel_with_tensor_memory_was_looked_at():
    assert sum("tmem_alloc" in body for _, body in kernels()) == 6
