"""Instructions of the kind that a whole warp executes together, read in the kernels' sources: its lanes meet (`__syncwarp`) wherever they may come from
loops of their own lengths.  Hardware need not join them by itself, and a barrier that part of a warp enters may never end."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_12637_b200", "csrc")


def _lines(name):
    """The lines that hold code, without their comments."""
    lines = [re.sub(r"//.*", "", line).strip() for line in open(os.path.join(CSRC, name))]
    return [line for line in lines if line]


def test_ahead_of_every_cluster_barrier():
    found = 0
    for path in glob.glob(os.path.join(CSRC, "*.cu*")):
        lines = _lines(os.path.basename(path))
        for before, line in zip(lines, lines[1:]):
            if "barrier.cluster" in line and ".aligned" in line:
                found += 1
                assert before == "__syncwarp();", (os.path.basename(path), line)
    assert found >= 3


def test_ahead_of_tensor_memory_taken_and_given_back():
    """Taking it follows zero fills and set-up that some of a warp's lanes do; where it does not end, neither does the block."""
    found = 0
    for path in glob.glob(os.path.join(CSRC, "*.cu*")):
        lines = _lines(os.path.basename(path))
        for before, line in zip(lines, lines[1:]):
            if re.search(r"tcgen05\.(alloc|dealloc)\.", line):
                found += 1
                assert before == "__syncwarp();", (os.path.basename(path), line)
    assert found == 4


def test_between_copies_and_matrix_instructions():
    """Rows that begin anywhere are copied in loops whose lanes take words of their own number."""
    for name in ("lbt_adapters.cu", "lbt_adapter_grads.cu"):
        text = " ".join(_lines(name))
        kernels = [k for k in text.split("__global__")[1:] if "copy_words<" in k]
        assert kernels
        for kernel in kernels:
            copies = kernel.rindex("copy_words<")
            product = min(at for at in (kernel.find(what, copies) for what in ("mma_step<", "rank_product<", "mma_split<")) if at >= 0)
            assert "__syncwarp();" in kernel[copies:product], (name, kernel[:200])
