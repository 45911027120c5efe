"""The 4-bit cache on the GPU, through the C ABI, against the fp64 forms of
tests/q4_ref.py: codes, scale bytes, counts and read-back values are equal bit for bit
(dividing by a power of two is exact, so a code is one rounding); attention outputs
lie within the bound that q4_ref.attend derives for them."""
import math

import numpy as np
import pytest
import torch

from paper_2609_25537_amd import cmc
from tests import q4_ref
from tests.gpu_util import DEV, say

pytestmark = pytest.mark.gpu

FLOAT = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t.to(dtype) if dtype is not None else t).to(DEV)


def host(t):
    return t.detach().cpu().to(torch.float64).numpy()


def raw(t):
    return t.detach().cpu().numpy()


def i32(x):
    return dev(np.asarray(x, np.int32))


def rows(rng, shape, kv="bf16", spread=0.5):
    """fp64 rows that the type holds exactly, channels of different sizes."""
    x = rng.standard_normal(shape) * np.exp(spread * rng.standard_normal(shape[-1]))
    return torch.from_numpy(x).to(FLOAT[kv]).to(torch.float64).numpy()


def filler(*shape):
    """Bytes that nothing may read: NaN scales."""
    return torch.full(shape, 255, dtype=torch.uint8, device=DEV)


def cache(B, H, R, Dh):
    return [filler(B, H, R, Dh // 2), filler(B, H, R, Dh // 2), filler(B, H, R, Dh // 32), filler(B, H, R, Dh // 32)]


def held(codes, scales):
    """Values as bf16 and fp32 hold them: all but those of 2^128 and up, which are infinite."""
    v = q4_ref.values(q4_ref.unpack(codes), np.asarray(scales).astype(np.int64))
    return np.where(np.abs(v) >= 2.0 ** 128, np.copysign(np.inf, v), v)


def quantised(x):
    """Packed codes and scale bytes of [..][Dh]."""
    c, s = q4_ref.quantise(x.reshape(-1, x.shape[-1]))
    d = x.shape[-1]
    return q4_ref.pack(c).reshape(*x.shape[:-1], d // 2), s.astype(np.uint8).reshape(*x.shape[:-1], d // 32)


# ------------------------------------------------------------------- codes

@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("e", [1, 90, 127, 200, 253])
def test_every_rounding(kv, e):
    """Every code, every midpoint between neighbours and both neighbours of it in fp32
    (bf16: in bf16), of either sign, under scale byte e."""
    say("codes", kv, e)
    c = q4_ref.MAGNITUDES
    x = np.concatenate([c, (c[1:] + c[:-1]) / 2]).astype(np.float32)
    step = np.float32(2.0 ** -8 if kv == "bf16" else 2.0 ** -23)
    x = np.concatenate([x, x * (1 + step), x * (1 - step), np.float32([1e-3, 2.0 ** -20])])
    x = np.concatenate([x, -x])
    x = x[np.abs(x) <= 6]
    n = -(-x.size // 31)
    x = np.concatenate([x, np.zeros(31 * n - x.size)]).reshape(n, 31)
    top = 3.0 if e == 253 else 6.0  # 6 * 2^126 passes fp32's range
    if e == 253:
        x = np.where(np.abs(x) <= 3, x, 0)
    pool = np.concatenate([np.full((n, 1), top), x], axis=1)
    if e == 253:
        pool[:, 0] = 3.25  # more than 6 of the scale below
    pool = np.ldexp(np.concatenate([pool, pool], axis=1), e - 127).reshape(1, 1, n, 64)
    t = dev(pool, FLOAT[kv])
    k4, v4, ks, vs = cmc.cmc_gather_tier1_q4(t, -t, None, n)
    want, s = q4_ref.quantise(host(t)[0, 0])
    assert (s == e).all() and (raw(ks) == e).all() and (raw(vs) == e).all()
    assert (raw(k4)[0, 0] == q4_ref.pack(want)).all() and (raw(v4)[0, 0] == q4_ref.pack(want ^ 8)).all()


SPECIAL = {
    "zeros": lambda x: x * 0,
    "negative zeros": lambda x: -(x * 0),
    "one large": lambda x: np.where(np.arange(x.size).reshape(x.shape) % 64 == 7, 3.4e38, x),
    "tiny": lambda x: x * 2.0 ** -130,
    "subnormal": lambda x: x * 2.0 ** -140,
    "infinities": lambda x: np.where(np.arange(x.size).reshape(x.shape) % 97 == 3, -np.inf, x),
    "all infinite": lambda x: np.full_like(x, np.inf),
    "nan": lambda x: np.where(np.arange(x.size).reshape(x.shape) % 89 == 5, np.nan, x),
    "nan and infinity": lambda x: np.where(np.arange(x.size).reshape(x.shape) % 5 == 0, np.nan, np.inf),
    "just over": lambda x: np.clip(x, -1, 1) * 6.01,
}


@pytest.mark.parametrize("what", sorted(SPECIAL))
@pytest.mark.parametrize("path", ["gather", "append", "prefill", "step"])
def test_special_values(what, path):
    say("special", what, path)
    rng = np.random.default_rng(3)
    R, Dh = 45, 64
    x = SPECIAL[what](rng.standard_normal((1, 2, R, Dh)))
    t = dev(x, torch.float32)
    x = host(t)
    want, wants = quantised(x)
    c = cache(1, 2, R, Dh)
    if path == "gather":
        cmc.cmc_gather_tier1_q4(t, t, None, R, out_k=c[0], out_v=c[1], out_ks=c[2], out_vs=c[3])
    else:
        count, step = i32([0]), R if path == "prefill" else 3
        q, tier = torch.randn(1, 4, Dh, device=DEV), cache(1, 2, 0, Dh)
        for n in range(0, R, step):
            new = t[:, :, n:n + step].contiguous()
            if path == "step":
                cmc.cmc_decode_step_q4(q, *tier, 0, *c, count, new, new, 0.1)
            else:
                cmc.cmc_window_append_q4(*c, count, new, new)
        assert count.item() == R
    for i in range(2):
        assert (raw(c[2 + i])[0] == wants[0]).all()
        assert (raw(c[i])[0] == want[0]).all()
    for dtype in FLOAT.values():
        k, v = cmc.cmc_cache_read_q4(*c, dtype=dtype)
        val = q4_ref.values(q4_ref.unpack(want), wants.astype(np.int64))
        val = torch.from_numpy(val).to(torch.float32).to(torch.float64).numpy()
        for y in (k, v):
            assert np.array_equal(host(y), val, equal_nan=True)
            finite = ~np.isnan(val)
            assert (np.signbit(host(y)) == np.signbit(val))[finite].all()


# -------------------------------------------------------- gather and append

@pytest.mark.parametrize("Dh,kv,k", [(128, "bf16", 77), (64, "f32", 33), (256, "f32", 130), (128, "f32", 1), (256, "bf16", 257),
                                     (64, "bf16", 128)])
@pytest.mark.parametrize("indexed", [False, True])
def test_gather(Dh, kv, k, indexed):
    say("gather", Dh, kv, k, indexed)
    rng = np.random.default_rng(k)
    B, H, N = 5, 3, k + 40
    pk, pv = rows(rng, (B, H, N, Dh), kv), rows(rng, (B, H, N, Dh), kv)
    idx = rng.integers(-3, N + 3, (B, k + 2)).astype(np.int32) if indexed else None  # out of range: clamped
    k_len = np.array([k, 0, -4, (k + 1) // 2, k + 9], np.int32)
    out = cache(B, H, k, Dh)
    cmc.cmc_gather_tier1_q4(dev(pk, FLOAT[kv]), dev(pv, FLOAT[kv]), None if idx is None else dev(idx), k, k_len=dev(k_len),
                            out_k=out[0], out_v=out[1], out_ks=out[2], out_vs=out[3])
    for i, pool in enumerate((pk, pv)):
        c, s = raw(out[i]), raw(out[2 + i])
        for b in range(B):
            n = min(max(int(k_len[b]), 0), k)
            at = np.clip(idx[b, :n], 0, N - 1) if indexed else np.arange(n)
            wc, ws = quantised(pool[b][:, at])
            assert (c[b, :, :n] == wc).all() and (s[b, :, :n] == ws).all()
            assert (c[b, :, n:] == 255).all() and (s[b, :, n:] == 255).all()  # left as they were


@pytest.mark.parametrize("B,H,Dh,W,kv", [(2, 3, 128, 70, "bf16"), (1, 1, 64, 5, "f32"), (3, 8, 256, 64, "f32"), (2, 2, 64, 33, "bf16")])
@pytest.mark.parametrize("how", ["append", "step"])
def test_append(B, H, Dh, W, kv, how):
    """Rows in calls of one to W, several times round the ring, one sequence's count
    below 0 at the start."""
    say("append", B, H, Dh, W, kv, how)
    rng = np.random.default_rng(W)
    c = cache(B, H, W, Dh)
    counts = [int(x) for x in rng.integers(0, 2 * W, B)]
    counts[0] = -3
    count = i32(counts)
    want = [raw(x).copy() for x in c]
    tier, q = cache(B, H, 0, Dh), torch.randn(B, 2 * H, Dh, device=DEV)
    for T in (1, W, 2, (W + 1) // 2, 1, W - 1 or 1, 3):
        T = min(T, W)
        nk, nv = rows(rng, (B, H, T, Dh), kv), rows(rng, (B, H, T, Dh), kv)
        tk, tv = dev(nk, FLOAT[kv]), dev(nv, FLOAT[kv])
        if how == "append":
            cmc.cmc_window_append_q4(*c, count, tk, tv)
        else:
            cmc.cmc_decode_step_q4(q, *tier, 0, *c, count, tk, tv, 0.1)
        for b in range(B):
            for h in range(H):
                q4_ref.append(want[0][b, h], want[2][b, h], counts[b], nk[b, h])
                n = q4_ref.append(want[1][b, h], want[3][b, h], counts[b], nv[b, h])
            counts[b] = n
        assert raw(count).tolist() == counts
        for x, w in zip(c, want):
            assert (raw(x) == w).all(), T


def test_append_one_and_many_launches_agree():
    """The same rows by one workgroup per sequence, by the larger launch, and by steps."""
    rng = np.random.default_rng(5)
    B, H, W, Dh, T = 2, 8, 96, 128, 12
    new = dev(rows(rng, (B, H, T, Dh)), torch.bfloat16)
    got = []
    for sizes in ((12,), (1,) * 12, (5, 7)):
        c, count, at = cache(B, H, W, Dh), i32([90, 7]), 0
        for n in sizes:
            part = new[:, :, at:at + n].contiguous()
            cmc.cmc_window_append_q4(*c, count, part, -part)
            at += n
        got.append([raw(x) for x in (*c, count)])
    for other in got[1:]:
        assert all((x == y).all() for x, y in zip(got[0], other))


def test_append_nothing_else_is_touched():
    c, count = cache(2, 2, 40, 128), i32([39, 4])
    new = torch.randn(2, 2, 2, 128, device=DEV)
    cmc.cmc_window_append_q4(*c, count, new, new)
    for x in c:
        left = raw(x) == 255
        assert left[0, :, 1:39].all() and left[1, :, :4].all() and left[1, :, 6:].all()


# --------------------------------------------------------------- read back

@pytest.mark.parametrize("Dh,R", [(128, 70), (64, 100), (256, 129), (256, 1)])
@pytest.mark.parametrize("kv", ["bf16", "f32"])
def test_read(Dh, R, kv):
    say("read", Dh, R, kv)
    rng = np.random.default_rng(R)
    counts = [R, 0, -2, max(1, R // 2), R + 1, 3 * R + R // 3, 2 ** 31 - 1]
    B, H = len(counts), 2
    codes, scales = rng.integers(0, 256, (2, B, H, R, Dh // 2)), rng.integers(1, 254, (2, B, H, R, Dh // 32))
    c = [dev(x.astype(np.uint8)) for x in (*codes, *scales)]
    for n in sorted({R, 1, (R + 1) // 2, 0}):
        out = [torch.full((B, H, n, Dh), 7.0, dtype=FLOAT[kv], device=DEV) for _ in range(2)]
        cmc.cmc_cache_read_q4(*c, count=i32(counts), rows=n, out_k=out[0], out_v=out[1])
        for i in range(2):
            val = held(codes[i], scales[i])
            for b in range(B):
                at = q4_ref.newest(R, counts[b], n)
                assert (host(out[i])[b, :, :len(at)] == val[b][:, at]).all()
                assert (host(out[i])[b, :, len(at):] == 7).all()
    k, v = cmc.cmc_cache_read_q4(*c, dtype=FLOAT[kv])  # no counts: all rows as they stand
    assert (host(k) == held(codes[0], scales[0])).all()
    k, v = cmc.cmc_cache_read_q4(*c, rows=1, dtype=FLOAT[kv])
    assert (host(v) == held(codes[1], scales[1])[:, :, -1:]).all()


def test_read_extreme_scales():
    """Foreign bytes: 0 (2^-127), 254 and 255 among them."""
    codes = torch.arange(256, dtype=torch.uint8, device=DEV).repeat(2).view(1, 1, 16, 32)
    for s in (0, 1, 2, 250, 253, 254, 255):
        scales = torch.full((1, 1, 16, 2), s, dtype=torch.uint8, device=DEV)
        want = held(raw(codes), raw(scales))
        for dtype in FLOAT.values():
            k, v = cmc.cmc_cache_read_q4(codes, codes, scales, scales, dtype=dtype)
            assert np.array_equal(host(k), want, equal_nan=True) and np.array_equal(host(v), want, equal_nan=True)


# --------------------------------------------------------------- attention

def make(rng, B, Hkv, R, Dh, spread=0.5, kspread=0.7):
    """A cache's arrays on the GPU and its fp64 values [2][B][Hkv][R][Dh]."""
    x = np.stack([rows(rng, (B, Hkv, R, Dh), "f32", s) for s in (kspread, spread)])
    t = [dev(y, torch.float32) for y in x]
    if R == 0:
        return cache(B, Hkv, 0, Dh), x
    c = cmc.cmc_gather_tier1_q4(*t, None, R)  # whose output other tests hold against the definition
    return list(c), np.stack([q4_ref.values(q4_ref.unpack(raw(c[i])), raw(c[2 + i]).astype(np.int64)) for i in range(2)])


def check(out, q, tier, ring, k_len, counts, scale, norm=True):
    """Every head's output against fp64 over its own list of keys."""
    got, qh = host(out), host(q)
    B, Hq, Dh = qh.shape
    Hkv = tier.shape[2]
    off = mag = 0.0
    for b in range(B):
        n, w = k_len[b], min(max(counts[b], 0), ring.shape[3])
        for h in range(Hq):
            kv = h // (Hq // Hkv)
            K, V = (np.concatenate([tier[i, b, kv, :n], ring[i, b, kv, :w]]) for i in range(2))
            want, bound = q4_ref.attend(qh[b, h], K, V, scale)
            err = np.abs(got[b, h] - want)
            assert (err <= bound).all(), (b, h, float((err / bound).max()))
            off, mag = off + float((err ** 2).sum()), mag + float((want ** 2).sum())
    # In the 2-norm the errors of a random list average out: what stays is exp2's argument,
    # of up to 32 in size, rounded to 2^-24 of itself, and sums of some hundred terms.
    if norm and mag > 0:
        assert math.sqrt(off / mag) <= 3e-6, math.sqrt(off / mag)


def attend(rng, B, Hq, Hkv, Dh, k, W, counts, k_len=None, scale=None, N=None, qmag=1.0, norm=True):
    say("q4 attend", B, Hq, Hkv, Dh, k, W, counts, k_len)
    N = k if N is None else N
    scale = Dh ** -0.5 if scale is None else scale
    tier, tv = make(rng, B, Hkv, N, Dh)
    ring, rv = make(rng, B, Hkv, W, Dh)
    q = torch.from_numpy(rng.standard_normal((B, Hq, Dh)) * qmag).to(torch.float32).to(DEV)
    for b in range(B):  # slots and rows that no list holds: NaN
        n = k if k_len is None else min(max(k_len[b], 0), k)
        w = min(max(counts[b], 0), W)
        for x in range(2):
            tier[x][b, :, n:] = 255
            tier[2 + x][b, :, n:] = 255
            ring[x][b, :, w:] = 255
            ring[2 + x][b, :, w:] = 255
    cnt = i32(counts)
    out = torch.full((B, Hq, Dh), math.nan, device=DEV)
    cmc.cmc_two_tier_decode_q4(q, *tier, k, *(ring if W else [None] * 4), cnt if W else None, scale,
                               k_len=None if k_len is None else i32(k_len), out=out)
    lens = [k] * B if k_len is None else [min(max(x, 0), k) for x in k_len]
    check(out, q, tv, rv, lens, counts, scale, norm)
    assert raw(cnt).tolist() == list(counts)
    return out


@pytest.mark.parametrize("Dh", [64, 128, 256])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("k,W", [(97, 150), (40, 0), (0, 130), (513, 900)])
def test_attend_shapes(Dh, G, k, W):
    attend(np.random.default_rng(Dh + G + k), 2, 3 * G, 3, Dh, k, W, [W, 3 * W + 1])


@pytest.mark.parametrize("k,W,counts,k_len", [
    (50, 70, [0, 1, 31, 32, 33, 69, 70, 71, -5], [0, 1, 50, 49, 32, -3, 60, 33, 0]),
    (1, 1, [0, 1, 5], [0, 1, 1]), (32, 32, [32, 31, 0], [32, 0, 31]), (64, 33, [33, 0, 34], None), (0, 5, [0, 2, 9], None),
])
def test_attend_counts(k, W, counts, k_len):
    out = attend(np.random.default_rng(k + W), len(counts), 8, 2, 128, k, W, counts, k_len, N=k + 3)
    for b, c in enumerate(counts):
        if c <= 0 and k_len is not None and k_len[b] <= 0:
            assert (out[b] == 0).all()  # an empty list


@pytest.mark.parametrize("B,Hkv,G,Dh,k,W", [
    (1, 8, 4, 128, 256, 512), (1, 8, 4, 128, 40, 6000), (3, 1, 8, 64, 7, 3000), (12, 8, 2, 64, 100, 200), (17, 8, 1, 128, 300, 100),
    (20, 8, 4, 64, 120, 300), (33, 8, 4, 128, 40, 130), (50, 8, 2, 128, 64, 64), (70, 8, 1, 64, 33, 95), (5, 13, 8, 256, 200, 700),
    (2, 4, 8, 256, 1000, 2000), (40, 1, 8, 256, 33, 500), (1, 1, 8, 128, 5000, 9000), (1, 1, 2, 64, 3, 20000), (1, 1, 1, 256, 200, 184),
    (1, 1, 1, 128, 0, 385), (20, 8, 8, 128, 500, 1100), (19, 8, 4, 64, 300, 700), (32, 8, 1, 256, 100, 2000), (33, 8, 4, 128, 100, 2000),
    (3, 1, 4, 64, 40, 120000), (1, 1, 8, 256, 0, 70000), (3, 1, 1, 64, 5000, 60000), (2, 2, 1, 128, 0, 40000),
])
def test_attend_plans(B, Hkv, G, Dh, k, W):
    rng = np.random.default_rng(B * Hkv)
    counts = [int(x) for x in rng.integers(0, 2 * W, B)]
    attend(rng, B, Hkv * G, Hkv, Dh, k, W, counts, [int(x) for x in rng.integers(0, k + 1, B)])


@pytest.mark.parametrize("scale", [-0.1, 0.0, 30.0, 1e-20])
def test_attend_logit_scales(scale):
    attend(np.random.default_rng(1), 2, 8, 2, 128, 60, 90, [90, 20], scale=scale, norm=abs(scale) < 1)


@pytest.mark.parametrize("mag", [0.0, 1e-38, 1e-30, 1e-6, 1e3])
@pytest.mark.parametrize("G", [1, 8])
def test_attend_query_sizes(mag, G):
    attend(np.random.default_rng(2), 2, 2 * G, 2, 64, 60, 90, [90, 20], qmag=mag, norm=mag < 1)


SHAPES = [(64, 1), (64, 4), (128, 2), (128, 4), (128, 8), (256, 1), (256, 8)]


@pytest.mark.parametrize("Dh,G", SHAPES)
def test_powers_of_two_between_q_k_and_scale(Dh, G):
    """The same scores with their size moved between q, K and the scale give the same
    outputs, bit for bit where nothing leaves fp32's range."""
    rng = np.random.default_rng(Dh + G)
    tier, tv = make(rng, 1, 2, 70, Dh)
    q = torch.from_numpy(rng.standard_normal((1, 2 * G, Dh))).to(torch.float32).to(DEV)
    base = cmc.cmc_two_tier_decode_q4(q, *tier, 70, None, None, None, None, None, 0.25)
    check(base, q, tv, np.zeros((2, 1, 2, 0, Dh)), [70], [0], 0.25)
    for dq, dk, ds in ((100, -100, 0), (-100, 100, 0), (-90, 0, 90), (90, 0, -90), (0, 100, -100), (0, -100, 100), (-60, 110, -50),
                       (-50, 100, -50), (50, -110, 60), (-120, 115, 5), (40, 60, -100)):
        moved = [tier[0], tier[1], tier[2] + dk if dk >= 0 else tier[2] - (-dk), tier[3]]
        out = cmc.cmc_two_tier_decode_q4(q * 2.0 ** dq, *moved, 70, None, None, None, None, None, 0.25 * 2.0 ** ds)
        if min(dq, dk, ds) > -115:
            assert torch.equal(out, base), (dq, dk, ds)
        else:  # q's own small elements are subnormal there
            check(out, q * 2.0 ** dq, np.stack([tv[0] * 2.0 ** dk, tv[1]]), np.zeros((2, 1, 2, 0, Dh)), [70], [0], 0.25 * 2.0 ** ds)


@pytest.mark.parametrize("Dh,G", SHAPES)
@pytest.mark.parametrize("sign", [1, -1])
def test_far_scores(Dh, G, sign):
    """Scores of 2^15 to 2^100 whose result does not hang on their rounding: one key
    far ahead of the others, or all keys equal."""
    rng = np.random.default_rng(Dh)
    n = 70
    for e in (15, 21, 22, 23, 24, 30, 60, 100):
        K = np.zeros((1, 1, n, Dh))
        K[:, :, :, 0] = 1.0
        K[:, :, 41, 0] = 2.0 if sign > 0 else 0.5
        V = rng.standard_normal((1, 1, n, Dh))
        c = list(cmc.cmc_gather_tier1_q4(dev(K, torch.float32), dev(V, torch.float32), None, n))
        val = q4_ref.values(q4_ref.unpack(raw(c[1])), raw(c[3]).astype(np.int64))[0, 0]
        q = torch.zeros(1, G, Dh, device=DEV)
        q[:, :, 0] = sign * 2.0 ** e * 1.37
        out = host(cmc.cmc_two_tier_decode_q4(q, *c, n, None, None, None, None, None, 1.0))
        assert np.abs(out - val[41]).max() <= 2.0 ** -20 * np.abs(val).max(), e
        K[:, :, 41, 0] = 1.0
        c = list(cmc.cmc_gather_tier1_q4(dev(K, torch.float32), dev(V, torch.float32), None, n))
        out = host(cmc.cmc_two_tier_decode_q4(q, *c, n, None, None, None, None, None, 1.0))
        assert np.abs(out - val.mean(axis=0)).max() <= 2.0 ** -18 * np.abs(val).max(), e


def test_values_of_extreme_rows():
    """V rows of scales from 2^-126 to 2^100: an output is exact to the rows that weigh."""
    rng = np.random.default_rng(8)
    for e in (-120, -60, 60, 100):
        tier, tv = make(rng, 1, 2, 60, 128)
        tier[3] = (tier[3].to(torch.int32) + e).clamp(1, 254).to(torch.uint8)
        tv[1] = q4_ref.values(q4_ref.unpack(raw(tier[1])), raw(tier[3]).astype(np.int64))
        q = torch.randn(1, 8, 128, device=DEV)
        out = cmc.cmc_two_tier_decode_q4(q, *tier, 60, None, None, None, None, None, 0.1)
        check(out, q, tv, np.zeros((2, 1, 2, 0, 128)), [60], [0], 0.1)


def test_nan_is_kept_where_it_is_attended():
    rng = np.random.default_rng(9)
    for G, Dh in ((1, 64), (4, 128), (8, 256)):
        for which in (2, 3):  # a K or a V scale
            tier, tv = make(rng, 2, 2, 40, Dh)
            ring, rv = make(rng, 2, 2, 40, Dh)
            q = torch.randn(2, 2 * G, Dh, device=DEV)
            tier[which][1, 0, 17, Dh // 32 - 1] = 255
            out = host(cmc.cmc_two_tier_decode_q4(q, *tier, 40, *ring, i32([40, 40]), 0.1))
            head = out[1, :G]
            assert np.isnan(head).all() if which == 2 else np.isnan(head[:, -32:]).all() and np.isfinite(head[:, :-32]).all()
            out[1, :G] = 0
            assert np.isfinite(out).all()


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("G", [2, 4, 8])
def test_a_query_head_that_is_not_finite_stays_alone(value, G):
    rng = np.random.default_rng(10)
    tier, _ = make(rng, 1, 2, 90, 128)
    q = torch.randn(1, 2 * G, 128, device=DEV)
    want = cmc.cmc_two_tier_decode_q4(q, *tier, 90, None, None, None, None, None, 0.1)
    q[0, 1, 5] = value
    out = cmc.cmc_two_tier_decode_q4(q, *tier, 90, None, None, None, None, None, 0.1)
    assert out[0, 1].isnan().all()
    out[0, 1] = want[0, 1]
    assert torch.equal(out, want)


def test_run_to_run():
    rng = np.random.default_rng(11)
    tier, _ = make(rng, 1, 8, 300, 128)
    ring, _ = make(rng, 1, 8, 700, 128)
    q, cnt = torch.randn(1, 32, 128, device=DEV), i32([700])
    ws = cmc.decode_workspace_q4(1, 32, 8, 128, 300, 700, DEV)
    first = cmc.cmc_two_tier_decode_q4(q, *tier, 300, *ring, cnt, 0.1, workspace=ws)
    for _ in range(5):
        assert torch.equal(cmc.cmc_two_tier_decode_q4(q, *tier, 300, *ring, cnt, 0.1, workspace=ws), first)


# -------------------------------------------------------------------- steps

@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hq,Hkv,Dh,k,W,counts", [
    (1, 32, 8, 128, 100, 200, [199]), (3, 4, 4, 64, 33, 50, [0, 47, 120]), (2, 16, 2, 256, 64, 70, [31, 64]),
    (9, 16, 8, 128, 20, 64, [0, 1, 30, 31, 32, 63, 64, 65, 500]), (40, 16, 8, 64, 10, 40, list(range(40))),
    (2, 8, 2, 128, 0, 3000, [2999, 100]), (1, 8, 1, 128, 2000, 40, [39]),
])
def test_step(kv, B, Hq, Hkv, Dh, k, W, counts):
    """Steps of 1, 3, 16 and 17 rows: the ring, the counts, and the attention over it."""
    rng = np.random.default_rng(B + W)
    tier, tv = make(rng, B, Hkv, k, Dh)
    ring, rv = make(rng, B, Hkv, W, Dh)
    cnt, ws = i32(counts), cmc.decode_workspace_q4(B, Hq, Hkv, Dh, k, W, DEV)
    want = [raw(x).copy() for x in ring]
    counts = list(counts)
    for T in (1, 3, 16, 17, 1):
        say("q4 step", kv, B, Hq, Hkv, Dh, k, W, T)
        new = [rows(rng, (B, Hkv, T, Dh), kv) for _ in range(2)]
        q = torch.from_numpy(rng.standard_normal((B, Hq, Dh))).to(torch.float32).to(DEV)
        out = cmc.cmc_decode_step_q4(q, *tier, k, *ring, cnt, *[dev(x, FLOAT[kv]) for x in new], Dh ** -0.5, workspace=ws)
        for b in range(B):
            for h in range(Hkv):
                for i in range(2):
                    n = q4_ref.append(want[i][b, h], want[2 + i][b, h], counts[b], new[i][b, h])
            counts[b] = n
        assert raw(cnt).tolist() == counts
        for x, w in zip(ring, want):
            assert (raw(x) == w).all()
        rv = np.stack([q4_ref.values(q4_ref.unpack(want[i]), want[2 + i].astype(np.int64)) for i in range(2)])
        check(out, q, tv, rv, [k] * B, counts, Dh ** -0.5)
        assert (ws[:4 * (B + B * Hkv)] == 0).all()  # counters ready for the next call


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("Dh,more", [(64, 0), (128, 0), (256, 0), (64, 1), (128, 1), (256, 1)])
@pytest.mark.parametrize("B,Hkv,G,k,W,counts", [(2, 2, 4, 40, 50, [45, 7]), (1, 2, 8, 500, 700, [1395]), (1, 1, 1, 0, 17, [16]),
                                               (41, 4, 2, 1500, 600, [599, 600, 0, 31, 1196])])
def test_step_of_as_many_rows_as_one_launch_takes(kv, Dh, more, B, Hkv, G, k, W, counts):
    """1024 / Dh rows, round the ring's end and over several workgroups' units, in four
    waves and in eight; and one more."""
    T = 1024 // Dh + more
    say("q4 step", kv, Dh, T, B, Hkv, G, k, W)
    rng = np.random.default_rng(T + W)
    tier, tv = make(rng, B, Hkv, k, Dh)
    ring, _ = make(rng, B, Hkv, W, Dh)
    counts = [counts[b % len(counts)] for b in range(B)]
    cnt = i32(counts)
    want = [raw(x).copy() for x in ring]
    new = [rows(rng, (B, Hkv, T, Dh), kv) for _ in range(2)]
    q = torch.from_numpy(rng.standard_normal((B, Hkv * G, Dh))).to(torch.float32).to(DEV)
    out = cmc.cmc_decode_step_q4(q, *tier, k, *ring, cnt, *[dev(x, FLOAT[kv]) for x in new], Dh ** -0.5)
    for b in range(B):
        for h in range(Hkv):
            for i in range(2):
                q4_ref.append(want[i][b, h], want[2 + i][b, h], counts[b], new[i][b, h])
        counts[b] += T
    assert raw(cnt).tolist() == counts
    for x, w in zip(ring, want):
        assert (raw(x) == w).all()
    rv = np.stack([q4_ref.values(q4_ref.unpack(want[i]), want[2 + i].astype(np.int64)) for i in range(2)])
    check(out, q, tv, rv, [k] * B, counts, Dh ** -0.5)


def test_step_fills_an_empty_ring_that_held_nan():
    """Slots never written hold NaN; the step's own rows are the only ones attended."""
    ring, cnt = cache(2, 2, 50, 128), i32([0, 0])
    q, new = torch.randn(2, 8, 128, device=DEV), torch.randn(2, 2, 2, 128, device=DEV)
    out = cmc.cmc_decode_step_q4(q, *cache(2, 2, 0, 128), 0, *ring, cnt, new, new, 0.1)
    assert out.isfinite().all() and raw(cnt).tolist() == [2, 2]


def test_step_without_a_ring():
    rng = np.random.default_rng(13)
    tier, tv = make(rng, 1, 2, 30, 64)
    q, new = torch.randn(1, 4, 64, device=DEV), torch.randn(1, 2, 1, 64, device=DEV)
    out = cmc.cmc_decode_step_q4(q, *tier, 30, *cache(1, 2, 0, 64), i32([4]), new, new, 0.1)
    check(out, q, tv, np.zeros((2, 1, 2, 0, 64)), [30], [0], 0.1)


def test_empty_batch():
    q = torch.empty(0, 8, 128, device=DEV)
    c = [torch.empty(0, 2, 4, n, dtype=torch.uint8, device=DEV) for n in (64, 64, 4, 4)]
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    new = torch.empty(0, 2, 1, 128, device=DEV)
    assert cmc.cmc_decode_step_q4(q, *c, 4, *c, none, new, new, 0.1).shape == (0, 8, 128)
    cmc.cmc_window_append_q4(*c, none, new, new)
    assert cmc.cmc_cache_read_q4(*c)[0].shape == (0, 2, 4, 128)
    assert cmc.cmc_gather_tier1_q4(new, new, None, 1)[0].shape == (0, 2, 1, 64)


@pytest.mark.parametrize("Hkv,Dh", [(1, 128), (3, 256)])
def test_offsets_past_32_bits(Hkv, Dh):
    """The longest caches: rows near their end are written, read back and attended where
    they lie (three heads of 256 are 6 GiB of codes an array, the last past 32 bits)."""
    R = 1 << 24
    say("longest 4-bit cache", Hkv, Dh)
    ring = [torch.zeros(1, Hkv, R, Dh // 2, dtype=torch.uint8, device=DEV) for _ in range(2)]
    ring += [torch.ones(1, Hkv, R, Dh // 32, dtype=torch.uint8, device=DEV) for _ in range(2)]
    cnt = i32([R - 3])
    new = torch.randn(1, Hkv, 3, Dh, device=DEV)
    cmc.cmc_window_append_q4(*ring, cnt, new[:, :, :2].contiguous(), new[:, :, :2].contiguous())
    q = 40 * new[:, :, 2].contiguous()  # far ahead of the zero rows
    last = new[:, :, 2:].contiguous()
    out = cmc.cmc_decode_step_q4(q, *cache(1, Hkv, 0, Dh), 0, *ring, cnt, last, last, 1.0)
    k, v = cmc.cmc_cache_read_q4(*ring, count=cnt, rows=3, dtype=torch.float32)
    assert cnt.item() == R
    zero = np.zeros((1, Dh))
    for h in range(Hkv):
        val = q4_ref.values(*q4_ref.quantise(host(new)[0, h]))
        assert (host(k)[0, h] == val).all() and (host(v)[0, h] == val).all()
        rows = np.concatenate([val, zero])
        want, bound = q4_ref.attend(host(q)[0, h], rows, rows, 1.0)
        assert (np.abs(host(out)[0, h] - want) <= bound + 1e-9).all()
    pool = torch.randn(1, Hkv, 8, Dh, device=DEV).to(torch.bfloat16)
    idx = torch.zeros(1, R, dtype=torch.int32, device=DEV)
    idx[0, -2:] = torch.tensor([5, 7])
    cmc.cmc_gather_tier1_q4(pool, pool, idx, R, out_k=ring[0], out_v=ring[1], out_ks=ring[2], out_vs=ring[3])
    for h in range(Hkv):
        wc, ws = quantised(host(pool)[0, h][[0, 5, 7]])
        assert (raw(ring[0][0, h, -3:]) == wc).all() and (raw(ring[3][0, h, -3:]) == ws).all()
