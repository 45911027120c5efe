"""The 8-bit decode over the ways its work is cut (splits, wave counts, the
append's own split), at sizes past what tests/test_gpu_cache8.py walks row by
row: caches of random codes and power-of-two scales, the reference in fp64 on the
device, the bound tests/q8_ref.py derives.  A step's ring is held against the
append's, bit for bit."""
import math

import numpy as np
import pytest
import torch

from paper_2609_25537_amd import cmc
from tests import q8_ref
from tests.gpu_util import DEV, say

pytestmark = pytest.mark.gpu

CODE = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}


def codes(gen, shape, code):
    b = torch.randint(-127, 128, shape, generator=gen, device=DEV, dtype=torch.int32).to(torch.int8)
    if code == "e4m3":  # 0x7f and 0xff are NaN: 0x7e instead
        b = torch.where((b == 127) | (b == -1), torch.full_like(b, 126), b)
    return b.view(CODE[code])


def scales(gen, shape, code):
    """Powers of two that bring values to about 1."""
    e = torch.randint(-2, 2, shape, generator=gen, device=DEV) - (8 if code == "e4m3" else 6)
    return torch.exp2(e.float())


def values(c, s, block):
    rows = torch.arange(c.shape[2], device=DEV) // block
    return c.to(torch.float32).to(torch.float64) * s.to(torch.float64)[:, :, rows, None]


def attend(q, K, V, live, scale):
    """fp64 outputs and their bound (q8_ref.attend) for q [B][Hkv][G][Dh], values
    [B][Hkv][n][Dh], live [B][n]."""
    q = q.to(torch.float64)
    z = scale * torch.matmul(q, K.transpose(2, 3).contiguous())
    z = z.masked_fill(~live[:, None, None, :], -math.inf)
    p = torch.softmax(z, dim=-1)
    want = torch.matmul(p, V)
    d, n = K.shape[3], live.sum(-1).to(torch.float64)[:, None, None]
    K = K * live[:, None, :, None]
    mags = abs(scale) * torch.matmul(q.abs(), K.abs().transpose(2, 3).contiguous())
    dz = mags * ((d + 8) * 2.0 ** -24 + 2.0 ** -21)
    dz = dz + abs(scale) * K.abs().sum(-1)[:, :, None, :] * q.abs().amax(-1, keepdim=True) * 2.0 ** -36
    top = z.masked_fill(~live[:, None, None, :], 0.0).abs().amax(-1)
    dz = dz.amax(-1) + 2.0 ** -22 * (top + 2)
    w = torch.expm1(2 * dz) + 2.0 ** -20 + (n + 64) * 2.0 ** -24
    bound = (torch.matmul(p, V.abs()) + want.abs()) * w[..., None]
    bound = bound + 2.0 ** -36 * (V * live[:, None, :, None]).abs().sum(2)[:, :, None, :]
    return want, bound + 1e-30


class Case:
    def __init__(self, B, Hkv, G, Dh, k, W, code="e4m3", block=32, seed=0, k_len=None, counts=None):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.B, self.Hkv, self.G, self.Dh, self.k, self.W, self.code, self.block, self.gen = B, Hkv, G, Dh, k, W, code, block, g
        self.pool = [codes(g, (B, Hkv, k, Dh), code) for _ in range(2)] + [scales(g, (B, Hkv, -(-k // block)), code) for _ in range(2)]
        self.win = [codes(g, (B, Hkv, W, Dh), code) for _ in range(2)] + [scales(g, (B, Hkv, -(-W // block)), code) for _ in range(2)]
        if counts is None:
            counts = [(W - 3, W + 5, 2 * W + W // 2, 1)[b % 4] for b in range(B)]
        self.count = torch.tensor(counts, dtype=torch.int32, device=DEV)
        self.k_len = None if k_len is None else torch.tensor(k_len, dtype=torch.int32, device=DEV)
        self.scale = 1 / math.sqrt(Dh)
        self.ws = cmc.decode_workspace_q8(B, Hkv * G, Hkv, Dh, k, W, DEV)

    def q(self):
        return torch.randn((self.B, self.Hkv * self.G, self.Dh), generator=self.gen, device=DEV)

    def new(self, T, dtype=torch.bfloat16):
        return [torch.randn((self.B, self.Hkv, T, self.Dh), generator=self.gen, device=DEV).to(dtype) for _ in range(2)]

    def check(self, q, out, win, count):
        kl = torch.full((self.B,), self.k, device=DEV) if self.k_len is None else self.k_len.clamp(0, self.k)
        live = torch.cat([torch.arange(self.k, device=DEV)[None] < kl[:, None],
                          torch.arange(self.W, device=DEV)[None] < count.clamp(0, self.W)[:, None]], 1)
        assert torch.isfinite(out).all()
        worst = 0.0
        for b in range(self.B):  # one sequence at a time: fp64 values take eight times the codes
            KV = [torch.cat([values(self.pool[x][b:b + 1], self.pool[2 + x][b:b + 1], self.block),
                             values(win[x][b:b + 1], win[2 + x][b:b + 1], self.block)], 2) for x in range(2)]
            qb = q[b:b + 1].view(1, self.Hkv, self.G, self.Dh)
            want, bound = attend(qb, KV[0], KV[1], live[b:b + 1], self.scale)
            err = (out[b:b + 1].view_as(want).to(torch.float64) - want).abs()
            worst = max(worst, float((err / bound).max()))
        assert worst <= 1.0, worst
        assert not self.ws[:4 * (self.B + self.B * self.Hkv)].any(), "arrival counters must return to zero"

    def attend(self):
        q = self.q()
        out = cmc.cmc_two_tier_decode_q8(q, *self.pool, self.k, *self.win, self.count, self.scale, self.block, k_len=self.k_len,
                                         workspace=self.ws)
        self.check(q, out, self.win, self.count)

    def step(self, T, dtype=torch.bfloat16):
        q, new = self.q(), self.new(T, dtype)
        ring = [t.clone() for t in (*self.win, self.count)]
        cmc.cmc_window_append_q8(*ring, *new, self.block)
        out = cmc.cmc_decode_step_q8(q, *self.pool, self.k, *self.win, self.count, *new, self.scale, self.block, k_len=self.k_len,
                                     workspace=self.ws)
        for x, y in zip((*self.win, self.count), ring):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        self.check(q, out, self.win, self.count)


PLANS = [
    # B, Hkv, G, Dh, k, W            pairs, units of 32 rows
    (1, 8, 4, 128, 256, 512),      # 8, 24: cut by the square root
    (5, 8, 4, 128, 2001, 1003),    # 40, 95
    (5, 8, 4, 128, 12003, 5001),   # 40, 533: 8 waves
    (8, 8, 2, 64, 9000, 8000),     # 64, 532: 8 waves
    (9, 8, 4, 128, 3001, 1502),    # 72, 141: an uneven number of splits
    (16, 8, 4, 128, 3001, 1502),   # 128, 141: 8 waves, half the splits
    (12, 8, 4, 128, 700, 333),     # 96, 33
    (12, 8, 4, 128, 200, 133),     # 96, 12
    (12, 8, 8, 256, 200, 133),     # 96, 12: many output registers
    (12, 8, 8, 256, 700, 333),     # 96, 33
    (19, 8, 4, 128, 1500, 700),    # 152, 69
    (19, 8, 4, 128, 1200, 500),    # 152, 54
    (19, 8, 4, 128, 300, 200),     # 152, 17
    (19, 8, 8, 256, 1200, 500),    # 152, 54
    (19, 8, 8, 256, 300, 200),     # 152, 17
    (25, 8, 4, 128, 700, 500),     # 200, 38: 8 waves
    (25, 8, 2, 64, 300, 200),      # 200, 17: 8 waves
    (25, 8, 4, 128, 300, 200),     # 200, 17
    (38, 8, 4, 128, 2500, 700),    # 304, 101: two splits
    (38, 8, 4, 128, 300, 200),     # 304, 17
    (50, 8, 1, 128, 300, 200),     # 400
]


@pytest.mark.parametrize("B,Hkv,G,Dh,k,W", PLANS)
def test_attend_plans(B, Hkv, G, Dh, k, W):
    for code, block in (("e4m3", 32), ("i8", 64)):
        say("8-bit attend", code, block, (B, Hkv, G, Dh, k, W))
        Case(B, Hkv, G, Dh, k, W, code, block, seed=B).attend()


@pytest.mark.parametrize("B,Hkv,G,Dh,k,W", PLANS)
def test_step_plans(B, Hkv, G, Dh, k, W):
    """One row, as many as the decode takes along, and more; ragged counts."""
    for code, block in (("e4m3", 32), ("i8", 128)):
        c = Case(B, Hkv, G, Dh, k, W, code, block, seed=B + 1, k_len=[(k, k // 2, 0, k + 1)[b % 4] for b in range(B)])
        for T in (1, 16, 17, 1):
            say("8-bit step", code, block, (B, Hkv, G, Dh, k, W), "T", T)
            c.step(T)


@pytest.mark.parametrize("code,dtype", [("e4m3", torch.float32), ("i8", torch.bfloat16)])
@pytest.mark.parametrize("B", [1, 12, 50])
def test_step_rows_over_three_blocks(code, dtype, B):
    """Sixteen rows that end one block, fill the short last one and begin the
    first again, and rings shorter than a block."""
    for W, block, counts in ((70, 32, [57] * B), (35, 32, [24] * B), (5, 32, [4] * B), (131, 64, [124 + 131] * B), (17, 128, [3] * B)):
        say("8-bit step over blocks", code, B, W, block)
        c = Case(B, 8, 4, 128, 40, W, code, block, seed=W, counts=counts)
        for T in (min(16, W), 1, min(15, W)):
            c.step(T, dtype)


def test_one_head_one_row():
    """The smallest calls: one head, one pool row or none, a ring of one slot."""
    for k, W in ((1, 1), (0, 1), (1, 2), (33, 1)):
        for Dh in (64, 128, 256):
            say("8-bit smallest", k, W, Dh)
            c = Case(1, 1, 1, Dh, k, W, "i8", 32, seed=W, counts=[0])
            if k:
                c.attend()
            for _ in range(3):
                c.step(1)


def test_codes_that_no_append_writes():
    """int8 -128, which the format's writers never make, counts as -128."""
    c = Case(2, 2, 2, 128, 70, 40, "i8", 32, seed=3, counts=[40, 7])
    for t in (c.pool[0], c.pool[1], c.win[0], c.win[1]):
        t[:, :, ::3, ::5] = -128
    c.attend()
    got_k, got_v = cmc.cmc_cache_read_q8(*c.win, 32, dtype=torch.float32)
    for got, x in ((got_k, 0), (got_v, 1)):
        assert torch.equal(got.to(torch.float64), values(c.win[x], c.win[2 + x], 32))


def test_gather_one_row_many_times():
    """An index list that names one row throughout, out of order ones, and ones
    past the pool (the last row)."""
    g = torch.Generator(device=DEV).manual_seed(5)
    B, H, N, Dh, k = 2, 3, 50, 128, 77
    pk, pv = (torch.randn((B, H, N, Dh), generator=g, device=DEV) for _ in range(2))
    idx = torch.full((B, k), 7, dtype=torch.int32, device=DEV)
    idx[1] = torch.arange(k, 0, -1, device=DEV, dtype=torch.int32) * 5 - 100
    out = cmc.cmc_gather_tier1_q8(pk, pv, idx, k, 32, dtype=torch.int8)
    at = idx.clamp(0, N - 1).long()[:, None, :, None].expand(B, H, k, Dh)
    for c, s, p in ((out[0], out[2], pk), (out[1], out[3], pv)):
        rows = torch.gather(p, 2, at).cpu().to(torch.float64).numpy()
        for b in range(B):
            for h in range(H):
                for j in range(-(-k // 32)):
                    want, ws = q8_ref.quantise(rows[b, h, 32 * j:32 * j + 32], "i8")
                    assert float(s[b, h, j]) == ws
                    assert np.array_equal(c[b, h, 32 * j:32 * j + 32].cpu().numpy(), want)


def test_step_of_many_rows_captured_and_replayed():
    """More rows than the decode takes along: an append and a decode in one graph."""
    c = Case(3, 8, 4, 128, 100, 70, seed=8)
    q, new, out = c.q(), c.new(20), torch.empty((3, 32, 128), device=DEV)
    start = [t.clone() for t in (*c.win, c.count)]
    ring = [t.clone() for t in start]

    def run(r, o):
        cmc.cmc_decode_step_q8(q, *c.pool, c.k, *r, *new, c.scale, c.block, out=o, workspace=c.ws)

    run(ring, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(ring, out)
    eager, want = [t.clone() for t in ring], torch.empty_like(out)
    for i in range(4):
        say("8-bit step of many rows: replay", i)
        q.mul_(0.9)
        graph.replay()
        run(eager, want)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        for x, y in zip(ring, eager):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        a = torch.randn(256, 256, device=DEV)
        (a @ a).sum().item()
    assert int(ring[4][0]) == int(start[4][0]) + 20 * 5


@pytest.mark.parametrize("e", [106, -126])
def test_values_of_extreme_blocks(e):
    """Values near 2^115, whose sums over the keys (and twice the binades that the
    running maximum may lag) fit fp32, and values at the smallest scale."""
    for Dh in (64, 128, 256):
        c = Case(2, 2, 2, Dh, 60, 50, "e4m3", 32, seed=e, counts=[50, 13])
        c.pool[3].fill_(2.0 ** e)
        c.win[3].fill_(2.0 ** e)
        c.attend()
        q = c.q()
        out = cmc.cmc_two_tier_decode_q8(q, *c.pool, c.k, *c.win, c.count, np.float32(c.scale), c.block, workspace=c.ws)
        assert torch.isfinite(out).all() and (out.abs().amax() > 2.0 ** e).item()


def test_a_query_head_that_is_not_finite_stays_alone():
    for what in (math.nan, math.inf, -math.inf):
        for G, Dh in ((4, 128), (8, 64), (2, 256)):
            c = Case(2, 2, G, Dh, 150, 70, "i8", 32, seed=G, counts=[70, 90])
            q = c.q()
            run = lambda: cmc.cmc_two_tier_decode_q8(q, *c.pool, c.k, *c.win, c.count, c.scale, c.block, workspace=c.ws)
            good = run()
            q[1, G, 5] = what
            bad = run()
            assert torch.isnan(bad[1, G]).all()
            keep = torch.ones(bad.shape[:2], dtype=torch.bool, device=DEV)
            keep[1, G] = False
            assert torch.equal(bad[keep], good[keep])
            assert not c.ws[:4 * (2 + 4)].any()


@pytest.mark.parametrize("code", ["e4m3", "i8"])
def test_scales_below_zero(code):
    """A cache made elsewhere whose scales have either sign, and logits of many
    binades: the largest score of a block may be its smallest product."""
    for Dh, G in ((64, 2), (128, 4), (256, 1)):
        c = Case(2, 4, G, Dh, 333, 150, code, 32, seed=Dh, counts=[150, 70])
        for s in (*c.pool[2:], *c.win[2:]):
            s.mul_(torch.where(torch.rand(s.shape, generator=c.gen, device=DEV) < 0.5, -1.0, 1.0))
        c.scale = 4.0
        c.attend()
        for kv, want_s in ((0, 2), (1, 3)):
            got = cmc.cmc_cache_read_q8(*c.win, 32, dtype=torch.float32)[kv]
            assert torch.equal(got.to(torch.float64), values(c.win[kv], c.win[want_s], 32))
