"""Every norm kernel in the library is one that some width and number of rows takes.

The rule is stated here once more (as few idle threads as there may be, fewer threads where that is equal) and gone through for
all widths; the kernels are the names that nm prints for the library that was built here."""
import re
import shutil
import subprocess

import pytest

from paper_2512_16843_b200 import binding as L


def choice(cols, rows_fill_the_sms):
    pieces, widest = cols // 8, 256 if rows_fill_the_sms else 512
    best = None
    for threads in (8, 16, 32, 64, 128, 256, 512):
        if threads > widest:
            break
        each = -(-pieces // threads)
        most = 3 if threads <= 32 else 8 if threads == 256 and rows_fill_the_sms else 4
        idle = threads * each - pieces
        if each <= most and (best is None or idle < best[0]):
            best = idle, threads, each
    return best[1:]


@pytest.mark.skipif(not shutil.which("nm"), reason="nm is not installed")
def test_no_kernel_that_no_call_takes():
    names = subprocess.run(["nm", "-C", L.LIB_PATH], capture_output=True, text=True, check=True).stdout
    built = {tuple(int(x) for x in m) for m in re.findall(r"::k_norm<(\d+), (\d+)u?, (\d)>\(", names)}
    taken = {choice(cols, fill) + (kind,) for cols in range(8, 16385, 8) for fill in (False, True) for kind in (L.NORM_NONE, L.NORM_LAYER, L.NORM_RMS)}
    assert built == taken
