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


@pytest.mark.parametrize("bar", ["bar_done", "bar_clear", "bar_bits"])
def test_one_lane_speaks_for_its_warp_after_a_warp_barrier(bar):
    """Long rows of the distillation loss: lane 0 arrives for what all lanes of its warp have stored or cleared.  Its release covers
    the others' accesses through a __syncwarp (a vote or shuffle orders no memory), else the named classes' gradient, which
    another warp writes over these stores, may come first."""
    with open(os.path.join(CSRC, "fw_distill_ring.cu")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    arrivals = re.findall(rf"([^;{{}}]*;)\s*if \(lane == 0\) sm100::mbar_arrive\(bar\({bar}\[", text)
    assert len(arrivals) == text.count(f"mbar_arrive(bar({bar}[") == 1
    assert arrivals[0].strip() == "__syncwarp();"
