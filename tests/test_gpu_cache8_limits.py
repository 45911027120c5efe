"""The 8-bit cache at the ends of fp32's range: scores far past what a model has,
against results that do not depend on how a score is rounded."""
import math

import numpy as np
import pytest
import torch

from paper_2609_25537_amd import cmc
from tests import q8_ref
from tests.gpu_util import DEV, say
from tests.test_gpu_cache8_plans import Case

pytestmark = pytest.mark.gpu

CODE = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}


def as_codes(x, code):
    """Tensors of whole numbers (e4m3: multiples of 8 up to 120) as codes."""
    return x.to(torch.float32).to(CODE[code])


class Far:
    """k Tier-1 rows and a full ring of W whose keys differ in their first dim
    alone: key t holds level[t] there, and the query `size` times a factor of its
    head's own in [1, 2)."""

    def __init__(self, level, k, Hkv, G, Dh, code, seed):
        B, n = 2, level.shape[-1]
        W = n - k
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.K = torch.zeros((B, Hkv, n, Dh), device=DEV)
        self.K[..., 0] = level
        self.V = 8.0 * torch.randint(-15, 16, (B, Hkv, n, Dh), generator=gen, device=DEV)
        self.B, self.Hkv, self.G, self.Dh, self.k, self.W = B, Hkv, G, Dh, k, W
        one = lambda r: torch.ones((B, Hkv, -(-r // 32)), device=DEV)
        cut = lambda x, a, b: as_codes(x[:, :, a:b].contiguous(), code)
        self.pool = [cut(self.K, 0, k), cut(self.V, 0, k), one(k), one(k)]
        self.win = [cut(self.K, k, n), cut(self.V, k, n), one(W), one(W)]
        self.count = torch.full((B,), W, dtype=torch.int32, device=DEV)
        self.factor = 1.0 + torch.rand((B, Hkv * G), generator=gen, device=DEV)
        self.ws = cmc.decode_workspace_q8(B, Hkv * G, Hkv, Dh, k, W, DEV)

    def query(self, size):
        q = torch.zeros((self.B, self.Hkv * self.G, self.Dh), device=DEV)
        q[..., 0] = self.factor * size
        return q

    def attend(self, q):
        return cmc.cmc_two_tier_decode_q8(q, *self.pool, self.k, *self.win, self.count, 0.125, 32, workspace=self.ws)


# log2 of the largest score (in units of log 2, a factor of 2 or so aside)
SIZES = [18, 20, 21, 22, 23, 24, 25, 26, 27, 28, 29, 30, 31, 32, 34, 40, 60, 100]
SHAPES = [(64, 1), (64, 8), (128, 4), (256, 2)]


@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("Dh,G", SHAPES)
@pytest.mark.parametrize("sign", [1, -1])
def test_far_scores_one_key(code, Dh, G, sign):
    """One key's score passes the others' by an eighth of itself at least, 2^15 and
    more: the output is its value.  Its weight is exact up to exp2's 2^-23, the
    sum's and the quotient's roundings come to less than 2^-21."""
    for at in (0, 37, 70, 129):  # in the pool, the ring, a unit of its own
        gen = torch.Generator(device=DEV).manual_seed(at)
        level = 8.0 * torch.randint(1, 8, (2, 3, 130), generator=gen, device=DEV)
        level[..., at] = 64.0
        if sign < 0:  # scores of -120 up to -64, and one of -56
            level = level - 128.0
            level[..., at] = -56.0
        c = Far(level, 60, 3, G, Dh, code, seed=at)
        want = c.V[:, :, at].repeat_interleave(G, dim=1)
        for size in SIZES:
            say("far scores", code, Dh, G, sign, "key", at, "2 **", size)
            out = c.attend(c.query(2.0 ** size / 64 / 0.125))
            assert ((out - want).abs() <= want.abs() * 2.0 ** -21).all(), (at, size)


@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("Dh,G", SHAPES)
@pytest.mark.parametrize("sign", [1, -1])
def test_far_scores_equal_keys(code, Dh, G, sign):
    """Keys that are all the same weigh the same: the mean of the values, off by
    the roundings of 130 terms' sums."""
    c = Far(torch.full((2, 3, 130), 40.0 * sign, device=DEV), 60, 3, G, Dh, code, seed=1)
    want = c.V.mean(2).repeat_interleave(G, dim=1)
    bound = c.V.abs().mean(2).repeat_interleave(G, dim=1) * (130 * 2.0 ** -24 + 2.0 ** -20)
    for size in SIZES:
        say("far scores, equal keys", code, Dh, G, sign, "2 **", size)
        out = c.attend(c.query(2.0 ** size / 40 / 0.125))
        assert ((out - want).abs() <= bound).all(), size


@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("Dh,G", SHAPES)
@pytest.mark.parametrize("sign", [1, -1])
def test_far_scores_a_rounding_apart(code, Dh, G, sign):
    """Scores that creep up (or down) by about a rounding from key to key, so that
    the maximum is passed by about its slack: whatever they weigh, equal values
    come out, off by the roundings of 130 terms' sums."""
    c = Far(torch.full((2, 3, 130), 64.0 * sign, device=DEV), 60, 3, G, Dh, code, seed=2)
    step = 8.0 * (torch.arange(130, device=DEV) // 9)  # 0 .. 112
    K = c.K.clone()
    K[..., 1] = step
    c.pool[0], c.win[0] = as_codes(K[:, :, :60].contiguous(), code), as_codes(K[:, :, 60:].contiguous(), code)
    for x in (c.pool[1], c.win[1]):
        x.copy_(as_codes(torch.full(x.shape, 88.0, device=DEV), code))
    for size in SIZES:
        for creep in (2.0, -2.0, 8.0):
            q = c.query(2.0 ** size / 64 / 0.125)
            q[..., 1] = creep * max(2.0 ** (size - 23), 1.0)
            say("far scores, close keys", code, Dh, G, sign, "2 **", size, creep)
            out = c.attend(q)
            assert ((out - 88.0).abs() <= 88.0 * (130 * 2.0 ** -24 + 2.0 ** -20)).all(), (size, creep)


@pytest.mark.parametrize("code", ["e4m3", "i8"])
def test_far_scores_in_a_step(code):
    """The appended row against the others, by the fused step and by one of more
    rows than it takes along."""
    for T in (1, 20):
        level = torch.full((2, 3, 130), 32.0, device=DEV)
        c = Far(level, 60, 3, 4, 128, code, seed=3)
        nk = torch.zeros((2, 3, T, 128), device=DEV)
        nv = 8.0 * torch.randint(-15, 16, (2, 3, T, 128), device=DEV)
        nv[..., 0] = 120.0  # the blocks' V scale stays 1 or a power of two below
        nk[:, :, -1, 0] = 64.0
        for size in (22, 26, 27, 30, 33):
            say("far scores, step", code, T, "2 **", size)
            out = cmc.cmc_decode_step_q8(c.query(2.0 ** size / 64 / 0.125), *c.pool, c.k, *c.win, c.count, nk, nv, 0.125, 32,
                                         workspace=c.ws)
            want = nv[:, :, -1].repeat_interleave(4, dim=1)
            # nv's codes: e4m3's own numbers, or whole numbers under a scale of 1 or below
            assert ((out - want).abs() <= want.abs() * 2.0 ** -21).all(), (T, size)
            c.count.fill_(c.W)


# ------------------------------------------------------------------ scales

@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("Dh,G", SHAPES)
@pytest.mark.parametrize("span", ["all", "small"])
def test_small_scales_of_a_foreign_cache(code, Dh, G, span):
    """V scales down to fp32's smallest normal numbers that are no powers of two.
    Keys of zeros make every weight the same, and values of one sign keep the mean's
    magnitude: sums of 130 terms, exp2 and the quotient are off by less than
    (130 + 16) 2^-24 of it."""
    gen = torch.Generator(device=DEV).manual_seed(Dh + G)
    c = Far(torch.zeros((2, 3, 130), device=DEV), 60, 3, G, Dh, code, seed=4)
    # every code above 0, or the least of them (e4m3: its subnormals, under scales that
    # leave the means normal numbers)
    top = 8 if span == "small" else 127
    floor = 2.0 ** -117 if code == "e4m3" and span == "small" else 2.0 ** -126
    b = torch.randint(1, top, (2, 3, 130, Dh), generator=gen, device=DEV, dtype=torch.int32).to(torch.int8)
    V = b.view(CODE[code])
    c.pool[1], c.win[1] = V[:, :, :60].contiguous(), V[:, :, 60:].contiguous()
    for e in (0, 1, 6, 12, 13, 14, 30):
        for s in (c.pool[3], c.win[3]):
            s.copy_((1.0 + torch.rand(s.shape, generator=gen, device=DEV)) * floor * 2.0 ** e)
        rows = lambda s, n: s.to(torch.float64)[:, :, torch.arange(n, device=DEV) // 32, None]
        v = V.to(torch.float32).to(torch.float64) * torch.cat([rows(c.pool[3], 60), rows(c.win[3], 70)], dim=2)
        want = v.mean(2).repeat_interleave(G, dim=1)
        say("small scales", code, Dh, G, span, e)
        out = c.attend(c.query(1.0)).to(torch.float64)
        assert ((out - want).abs() <= want * (130 + 16) * 2.0 ** -24).all(), e


# ------------------------------------------------------------------ values

def host(t):
    return t.detach().cpu().to(torch.float64).numpy()


@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("Dh,block", [(64, 32), (256, 128)])
@pytest.mark.parametrize("path,T", [("append", 1), ("append", 3), ("step", 1), ("step", 5), ("append", 40)])
def test_rings_of_the_largest_values(code, Dh, block, path, T):
    """Elements up to fp32's largest, whose codes stand for 2^128, and infinities,
    whose codes stand for more, keep their block's scale until they are evicted,
    and their codes where only the other array's scale moves."""
    H, W = 2, 40
    rng = np.random.default_rng(T)
    n = -(-W // block)
    most = float(np.finfo(np.float32).max)
    fresh = lambda: torch.zeros((1, H, W, Dh), dtype=torch.int8, device=DEV).view(CODE[code])
    ring = [fresh(), fresh(), torch.zeros((1, H, n), device=DEV), torch.zeros((1, H, n), device=DEV)]
    count = torch.zeros((1,), dtype=torch.int32, device=DEV)
    model = [(np.zeros((H, W, Dh)), np.zeros((H, n))) for _ in range(2)]
    pool = [torch.zeros((1, H, 8, Dh), dtype=torch.int8, device=DEV).view(CODE[code]), torch.ones((1, H, 1), device=DEV)]
    q = torch.zeros((1, H, Dh), device=DEV)
    seen, step = 0, 0
    while seen < 3 * W:
        nk = rng.standard_normal((1, H, T, Dh)) * 1.5 ** step  # K's scale moves every other time
        nv = rng.standard_normal((1, H, T, Dh)) * 1e37
        if step == 0:
            nv[0, 0, 0, :8] = [most, -most, np.inf, -np.inf, 3.3e38, -3.37e38, 2.5e38, 0.96875 * 2.0 ** 128]
            nv[0, 1, 0, :3] = [np.inf, 3e38, -1e-3]
        nk, nv = nk.astype(np.float32), nv.astype(np.float32)
        dk, dv = (torch.from_numpy(x).to(DEV) for x in (nk, nv))
        say("largest values", code, Dh, block, path, T, "row", seen)
        if path == "append":
            cmc.cmc_window_append_q8(*ring, count, dk, dv, block)
        else:
            cmc.cmc_decode_step_q8(q, pool[0], pool[0], pool[1], pool[1], 8, *ring, count, dk, dv, 0.1, block)
        for x, new in enumerate((nk, nv)):
            c, s = model[x]
            for h in range(H):
                q8_ref.append(c[h], s[h], seen, new[0, h].astype(np.float64), code, block)
            assert (host(ring[2 + x])[0] == s).all(), (seen, x)
            assert (host(ring[x])[0] == c).all(), (seen, x)
        seen += T
        step += 1
        assert int(count) == seen
    assert model[1][1].max() < 2.0 ** (120 if code == "e4m3" else 122)  # the large ones are gone


@pytest.mark.parametrize("R", [1 << 26, (1 << 26) - 3])
def test_read_back_of_the_longest_cache(R):
    """As many rows as a cache may have, of 256 to fp32: more threads than a launch
    holds in one dimension."""
    torch.cuda.empty_cache()
    Dh = 256
    k8 = torch.zeros((1, 1, R, Dh), dtype=torch.int8, device=DEV)
    scale = torch.ones((1, 1, -(-R // 128)), device=DEV)
    k8[0, 0, 0], k8[0, 0, R - 1], k8[0, 0, R // 2] = 5, 7, 9
    scale[0, 0, -1] = 0.5
    count = torch.full((1,), R, dtype=torch.int32, device=DEV)
    out = torch.empty((1, 1, R, Dh), device=DEV)
    say("longest cache", R)
    # K and V alike, into the same place: 64 GiB of output instead of 128
    cmc.cmc_cache_read_q8(k8, k8, scale, scale, 128, count=count, out_k=out, out_v=out)
    for at, want in ((0, 5.0), (1, 0.0), (R // 2, 9.0), (R - 2, 0.0), (R - 1, 3.5)):
        assert (out[0, 0, at] == want).all(), at
    assert float(out[0, 0, R - 4096:].sum(dtype=torch.float64)) == 3.5 * Dh
    out[0, 0, :8] = -1.0
    count.fill_(3)  # three live rows: nothing else is written
    cmc.cmc_cache_read_q8(k8, k8, scale, scale, 128, count=count, out_k=out, out_v=out)
    assert (out[0, 0, 0] == 5).all() and (out[0, 0, 1:3] == 0).all() and (out[0, 0, 3:8] == -1).all()
    count.fill_(R + 1)  # wrapped by one: the oldest is row 1
    cmc.cmc_cache_read_q8(k8, k8, scale, scale, 128, count=count, out_k=out, out_v=out)
    assert (out[0, 0, R - 1] == 5).all() and (out[0, 0, R - 2] == 3.5).all() and (out[0, 0, 0] == 0).all()
    del k8, out
    torch.cuda.empty_cache()


# ---------------------------------------------------------------- products

@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("Dh,G", SHAPES)
def test_powers_of_two_between_q_k_and_scale(code, Dh, G):
    """K's scales times 2^a, q times 2^b and scale times 2^-(a + b) leave the scores
    as they are: the same bits out, however small or large each of them is.  (A q
    below 2^-111 is held with other parts: within the bound.)"""
    c = Case(2, 2, G, Dh, 333, 150, code, 32, seed=Dh, counts=[150, 70])
    q = c.q()
    run = lambda q: cmc.cmc_two_tier_decode_q8(q, *c.pool, c.k, *c.win, c.count, c.scale, c.block, workspace=c.ws)
    want = run(q)
    c.check(q, want, c.win, c.count)
    ks = [t.clone() for t in (c.pool[2], c.win[2])]
    base = c.scale
    for a, b in ((126, -100), (120, -100), (100, -60), (126, -20), (-110, 100), (-110, -10), (100, 0), (60, 40), (-60, -60),
                 (126, -118), (110, -124)):
        say("powers", code, Dh, G, a, b)
        for t, s in zip((c.pool[2], c.win[2]), ks):
            t.copy_(s * 2.0 ** a)
        c.scale = base * 2.0 ** -(a + b)
        qb = q * 2.0 ** b
        out = run(qb)
        if b >= -104:
            assert torch.equal(out, want), (a, b, float((out - want).abs().max()))
        else:
            c.check(qb, out, c.win, c.count)
