"""A kernel that takes tensor memory waits for the kernels before it first.

Blocks of a kernel may start while blocks of its predecessor still run (programmatic launch).  Tensor memory is handed out per
SM and its allocation waits without a bound; a block that held columns while it waits for the predecessor's end, beside
a block of the predecessor that still needs some, would never go on.  Read from the sources: nothing runs on a GPU."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_16843_b200", "csrc")


def kernels():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        starts = [m.start() for m in re.finditer(r"__global__", text)] + [len(text)]
        for a, b in zip(starts, starts[1:]):
            body = text[a:b]
            name = re.search(r"(k_\w+)\s*\(", body)
            if "tcgen05.alloc" in body:
                yield os.path.basename(path), name.group(1), body


def test_all_kernels_with_tensor_memory_are_found():
    found = {name for _, name, _ in kernels()}
    assert {"k_attn_tc", "k_attn_weights", "k_scan_tc"} <= found and len(found) >= 5


@pytest.mark.parametrize("file,name,body", list(kernels()), ids=lambda x: x if isinstance(x, str) and len(x) < 40 else "")
def test_tensor_memory_is_taken_behind_the_wait(file, name, body):
    assert 0 <= body.find("griddep_sync()") < body.find("tcgen05.alloc"), (file, name)
