"""What the header says of the steps' launches, against the constants that decide them."""
import os
import re

from paper_2609_25537_amd import build


def _read(*path):
    with open(os.path.join(*path)) as f:
        return f.read()


def _comment_of(name):
    """The comment before a declaration of include/cmc.h, on one line."""
    src = _read(build.INCLUDE, "cmc.h")
    head = src[:re.search(rf"^cmc_status {name}\(", src, re.M).start()]
    return re.sub(r"\s+\*?\s*", " ", head[head.rindex("/*"):])


def test_rows_that_a_step_appends_in_its_launch():
    k = _read(build.CSRC, "kernels.hpp")
    rows8 = re.search(r"constexpr int kFusedRows8 = (\d+);", k)[1]
    assert f"in a single launch for up to {rows8} rows." in _comment_of("cmc_decode_step_q8")
    rows4 = re.search(r"constexpr int fused_rows4\(int Dh\) \{ return 4 \* 64 / 2 \* (\d+) / Dh; \}", k)[1]
    assert f"in a single launch for up to {4 * 64 // 2 * int(rows4)} / Dh rows." in _comment_of("cmc_decode_step_q4")
