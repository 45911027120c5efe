"""How the 4-bit decode's work is cut, on the CPU: the library's own plan over batches and
lengths."""
import ctypes

import pytest

from paper_2609_25537_amd import cmc

UNIT = 32  # rows


class Plan(ctypes.Structure):  # DecodePlan of csrc/kernels.hpp
    _fields_ = [("S", ctypes.c_int), ("chunk", ctypes.c_int), ("waves", ctypes.c_int), ("own_append", ctypes.c_bool),
                ("counter_bytes", ctypes.c_size_t), ("ml_bytes", ctypes.c_size_t), ("acc_bytes", ctypes.c_size_t),
                ("total", ctypes.c_size_t)]


def plan(pairs, units, G=4, Dh=128):
    f = cmc.lib()["_ZN3cmc12plan_decode4Eiiiiii"]  # cmc::plan_decode4(B, Hq, Hkv, Dh, k, W)
    f.argtypes, f.restype = [ctypes.c_int] * 6, Plan
    pool = units // 3
    return f(pairs, G, 1, Dh, pool * UNIT, (units - pool) * UNIT)


HEADS = [(64, 1), (64, 8), (128, 1), (128, 4), (128, 8), (256, 1), (256, 4), (256, 8)]


def waves(pairs, units, G, Dh):
    """Of a pair's whole axis, as measured: where eight waves cost more than they save a
    workgroup has four."""
    if Dh == 256:
        least = 48 if G == 8 else 64
    else:
        least = 40 if Dh == 128 and G < 8 and pairs > 208 else 12
    return 8 if pairs <= 256 and units >= least else 4


@pytest.mark.parametrize("Dh,G", HEADS)
def test_waves_of_whole_axes(Dh, G):
    """Short lists of wide heads, and of heads of 128 where nearly every CU has a workgroup,
    stay with four waves; other lists from 12 units on have eight."""
    for units in (1, 11, 12, 13, 14, 20, 39, 40, 47, 48, 63, 64, 144, 1026):
        for pairs in [*range(1, 129), *range(160, 270)]:
            p = plan(pairs, units, G, Dh)
            if p.S == 1:
                assert p.waves == waves(pairs, units, G, Dh), (pairs, units)


@pytest.mark.parametrize("Dh,G", HEADS)
def test_waves_of_batches_too_large_to_split(Dh, G):
    """129 pairs and more have one workgroup each: the same waves as 160 have."""
    for units in (12, 13, 14, 40, 48, 64, 144, 500):
        for pairs in range(129, 161):
            p = plan(pairs, units, G, Dh)
            assert (p.S, p.waves) == (1, waves(pairs, units, G, Dh)), (pairs, units)


@pytest.mark.parametrize("units", [1, 2, 11, 12, 13, 14, 24, 25, 48, 144, 145, 500, 1026, 4096])
def test_plans_cover_the_axis(units):
    """Splits of whole turns of their waves, every one with units, the partials within what the
    workspace query asks for."""
    for pairs in (1, 2, 7, 8, 31, 64, 65, 96, 127, 128, 129, 136, 152, 159, 160, 192, 256, 257, 512, 4096):
        for G, Dh in ((1, 64), (4, 128), (8, 256)):
            p = plan(pairs, units, G, Dh)
            assert p.waves in (4, 8) and 1 <= p.S <= 127 and p.chunk % p.waves == 0
            assert (p.S - 1) * p.chunk < units <= p.S * p.chunk
            parts = pairs * p.S * G * 4 if p.S > 1 else 0
            assert p.ml_bytes >= 2 * parts and p.acc_bytes >= Dh * parts and p.counter_bytes >= 8 * pairs
            assert p.total == p.counter_bytes + p.ml_bytes + p.acc_bytes
            pool = units // 3
            assert p.total == cmc.cmc_decode_q4_workspace_bytes(pairs, G, 1, Dh, pool * UNIT, (units - pool) * UNIT)
