"""What the header says of the steps' launches, against the constants that decide them."""
import os
import re

import numpy as np

from paper_2609_25537_amd import build


def _read(*path):
    with open(os.path.join(*path)) as f:
        return f.read()


def _comment_of(name):
    """The comment before a declaration of include/cmc.h, on one line."""
    src = _read(build.INCLUDE, "cmc.h")
    head = src[:re.search(rf"^cmc_status {name}\(", src, re.M).start()]
    return re.sub(r"\s+", " ", re.sub(r"\n \*", " ", head[head.rindex("/*"):]))


def test_rows_that_a_step_appends_in_its_launch():
    k = _read(build.CSRC, "kernels.hpp")
    rows8 = re.search(r"constexpr int kFusedRows8 = (\d+);", k)[1]
    assert f"in a single launch for up to {rows8} rows." in _comment_of("cmc_decode_step_q8")
    rows4 = re.search(r"constexpr int fused_rows4\(int Dh\) \{ return 4 \* 64 / 2 \* (\d+) / Dh; \}", k)[1]
    assert f"in a single launch for up to {4 * 64 // 2 * int(rows4)} / Dh rows." in _comment_of("cmc_decode_step_q4")


def test_accuracy_of_the_rotations_angles():
    """The kernel's turns are pos * (inv_freq * c) with c = fp64(1 / 2 pi): three roundings, so
    3 * 2^-53 at most, and more than 2^-52 for some.  long double has 64 bits."""
    assert np.finfo(np.longdouble).nmant >= 63
    src = _read(build.CSRC, "rope.hip")
    c = re.search(r"\(double\)p\.pos\[token\] \* \(\(double\)p\.inv_freq\[i\] \* (0\.1591\d+)\)", src)[1]
    rng = np.random.default_rng(0)
    pos = rng.integers(-2 ** 31, 2 ** 31, 400000)
    freq = np.exp(rng.uniform(np.log(1e-7), 0, pos.size)).astype(np.float32)
    got = pos.astype(np.float64) * (freq.astype(np.float64) * np.float64(c))
    want = pos.astype(np.longdouble) * freq.astype(np.longdouble) * np.longdouble("0.15915494309189533576888376337251436203")
    off = float(np.abs((got.astype(np.longdouble) - want) / want).max())
    for text, says in ((_comment_of("cmc_norm_rope"), r"pos \* inv_freq to 2\^-(\d+) of itself"),
                       (src, r"pos \* inv_freq is right to\s+// 2\^-(\d+) of itself")):
        assert off <= 2.0 ** -int(re.search(says, text)[1])
    assert off <= 3 * 2.0 ** -53
