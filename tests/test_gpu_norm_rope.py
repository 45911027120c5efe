"""cmc_norm_rope on the GPU against fp64: the norm, the rotation and where the results
lie; and the flow from a projection through a 4-bit cache to the attention, eager,
captured and on two streams."""
import math

import numpy as np
import pytest
import torch

from paper_2609_25537_amd import cmc
from tests import q4_ref
from tests.gpu_util import DEV, say

pytestmark = pytest.mark.gpu

FLOAT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a step


def host(t):
    return t.detach().cpu().to(torch.float64).numpy()


def reference(x, pos, inv_freq, weight, eps, interleaved):
    """x [B][T][H][Dh] fp64 -> the result, and an entrywise bound of what fp32 may be off:
    a square sum of Dh terms, its root, two products and the rotation's products and sum
    (a handful of 2^-24 of the pair's size), sines and cosines to 2^-22."""
    Dh, rot = x.shape[-1], 2 * inv_freq.size
    if weight is not None:
        with np.errstate(divide="ignore", invalid="ignore"):
            x = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * weight
    t = pos[..., None, None].astype(np.float64) * inv_freq.astype(np.float64)
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    y, size = x.copy(), np.abs(x)
    y[..., a] = x[..., a] * np.cos(t) - x[..., b] * np.sin(t)
    y[..., b] = x[..., b] * np.cos(t) + x[..., a] * np.sin(t)
    size[..., a] = size[..., b] = np.hypot(x[..., a], x[..., b])
    # the angle's own rounding in fp64, where a position is large
    far = np.zeros_like(y)
    far[..., a] = far[..., b] = np.abs(t) * 2.0 ** -51
    err = (0.0 if weight is None else (math.log2(Dh) + 8) * 2.0 ** -24) + (2.0 ** -21 if rot else 0.0) + far
    return y, size * err + 1e-44


def check(got, want, bound, kind):
    got, ok = host(got), np.isfinite(want)
    assert (np.isnan(got) == np.isnan(want)).all() and (got[~ok & ~np.isnan(want)] == want[~ok & ~np.isnan(want)]).all()
    tol = bound * 1.01 + np.abs(want) * EPS[kind] * 1.01 + (1e-40 if kind == "bf16" else 0)
    err = np.abs(got - want)[ok]
    assert (err <= tol[ok]).all(), float((err / tol[ok]).max())


def projection(rng, B, T, Hq, Hkv, Dh, kind, spread=0.5):
    x = rng.standard_normal((B, T, Hq + 2 * Hkv, Dh)) * np.exp(spread * rng.standard_normal((Hq + 2 * Hkv, Dh)))
    x = torch.from_numpy(x).to(FLOAT[kind]).to(DEV)
    return x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]


def freqs(rot, base=10000.0):
    f = (base ** (-np.arange(0, rot, 2) / max(rot, 1))).astype(np.float32)
    return f, torch.from_numpy(f).to(DEV)


def run(rng, B, T, Hq, Hkv, Dh, rot, kind, norm, interleaved, q_to="f32", kv_to="bf16", pos=None, eps=1e-6, q=None, k=None, v=None):
    say("rope", B, T, Hq, Hkv, Dh, rot, kind, norm, interleaved, q_to, kv_to)
    if q is None:
        q, k, v = projection(rng, B, T, Hq, Hkv, Dh, kind)
    pos = rng.integers(0, 40000, (B, T)) if pos is None else pos
    f, tf = freqs(rot)
    w = [(1 + 0.3 * rng.standard_normal(Dh)).astype(np.float32) if norm else None for _ in range(2)]
    tw = [None if x is None else torch.from_numpy(x).to(DEV) for x in w]
    tp = torch.from_numpy(pos.astype(np.int32)).to(DEV)
    oq, ok, ov = cmc.cmc_norm_rope(q, k, v, tp, tf, q_weight=tw[0], k_weight=tw[1], eps=eps, interleaved=interleaved,
                                   q_dtype=FLOAT[q_to], kv_dtype=FLOAT[kv_to])
    w = [None if x is None else x.astype(np.float64) for x in w]
    check(oq, *reference(host(q), pos, f, w[0], np.float32(eps), interleaved), q_to)
    want, bound = reference(host(k), pos, f, w[1], np.float32(eps), interleaved)
    check(ok, want.swapaxes(1, 2), bound.swapaxes(1, 2), kv_to)
    want = torch.from_numpy(host(v)).to(FLOAT[kv_to]).to(torch.float64).numpy().swapaxes(1, 2)
    assert np.array_equal(host(ov), want, equal_nan=True)  # laid out, rounded once
    return oq, ok, ov


@pytest.mark.parametrize("Dh,rot", [(64, 64), (64, 16), (128, 128), (128, 64), (128, 48), (256, 256), (256, 240), (256, 0), (64, 0)])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_shapes(Dh, rot, kind, interleaved, norm):
    rng = np.random.default_rng(Dh + rot)
    run(rng, 2, 5, 6, 3, Dh, rot, kind, norm, interleaved, q_to="f32" if rot % 32 else "bf16", kv_to=kind)


@pytest.mark.parametrize("B,T,Hq,Hkv", [(1, 1, 32, 8), (64, 1, 32, 8), (1, 1, 1, 1), (3, 1, 64, 8), (1, 2051, 4, 2), (5, 700, 3, 1),
                                        (2, 1024, 8, 8), (2047, 1, 2, 1), (2048, 1, 1, 1)])
def test_sizes(B, T, Hq, Hkv):
    run(np.random.default_rng(B * T), B, T, Hq, Hkv, 128, 128, "bf16", True, False)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(interleaved):
    """Positions to the ends of int32, negative ones among them."""
    rng = np.random.default_rng(4)
    pos = np.array([[0, 1, -1, 2 ** 20, 2 ** 20 + 1, 10 ** 7, -10 ** 7, 2 ** 31 - 1, -2 ** 31]])
    run(rng, 1, pos.size, 2, 2, 128, 128, "f32", False, interleaved, kv_to="f32", pos=pos)


@pytest.mark.parametrize("mag", [0.0, 1e-44, 1e-38, 1e-30, 1e-21, 1e-19, 1e10, 1e18, 1e19, 1e30, 3e38])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6])
def test_row_sizes(mag, eps):
    """Rows whose squares leave fp32's range on either side."""
    rng = np.random.default_rng(5)
    x = torch.from_numpy(rng.uniform(-1, 1, (1, 3, 4, 64)) * mag).to(torch.float32).to(DEV)
    run(rng, 1, 3, 4, 4, 64, 32, "f32", True, False, kv_to="f32", eps=eps, q=x, k=x, v=x)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("norm", [False, True])
def test_not_finite(value, norm):
    """It stays in its head; without a norm, in its pair."""
    rng = np.random.default_rng(6)
    q, k, v = projection(rng, 1, 3, 4, 2, 128, "f32")
    want = run(rng, 1, 3, 4, 2, 128, 64, "f32", norm, False, kv_to="f32", q=q, k=k, v=v)
    rng = np.random.default_rng(6)
    projection(rng, 1, 3, 4, 2, 128, "f32")
    q = q.clone()
    q[0, 1, 2, 5] = value
    f, tf = freqs(64)
    pos = rng.integers(0, 40000, (1, 3))
    tw = [torch.from_numpy((1 + 0.3 * rng.standard_normal(128)).astype(np.float32)).to(DEV) if norm else None for _ in range(2)]
    oq, _, _ = cmc.cmc_norm_rope(q, k, v, torch.from_numpy(pos.astype(np.int32)).to(DEV), tf, q_weight=tw[0], k_weight=tw[1])
    bad = ~oq.isfinite()
    assert bad[0, 1, 2].any()
    if norm:
        if math.isinf(value):  # x / inf: zeros, and NaN where the infinity was
            oq[0, 1, 2] = want[0][0, 1, 2]
        else:
            assert oq[0, 1, 2].isnan().all()
    else:
        assert bad[0, 1, 2].nonzero().flatten().tolist() == [5, 37]
    oq[0, 1, 2] = want[0][0, 1, 2]
    assert torch.equal(oq, want[0])


@pytest.mark.parametrize("value", [math.inf, -math.inf])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved,dim,pair", [(False, 5, [5, 37]), (False, 37, [5, 37]), (False, 100, [100]), (True, 5, [4, 5]),
                                                  (True, 62, [62, 63]), (True, 64, [64])])
def test_an_infinity_under_a_norm(value, kind, interleaved, dim, pair):
    """x / sqrt(infinity): NaN where the infinity was, 0 elsewhere in its head, and the NaN
    in both dims of its pair where that one turns; no other head changes."""
    say("rope infinity", value, kind, interleaved, dim)
    rng = np.random.default_rng(16)
    q, k, v = (x.clone() for x in projection(rng, 2, 3, 4, 2, 128, kind))
    f, tf = freqs(64)
    pos = torch.from_numpy(rng.integers(1, 40000, (2, 3)).astype(np.int32)).to(DEV)
    how = dict(q_weight=torch.from_numpy((1 + 0.3 * rng.standard_normal(128)).astype(np.float32)).to(DEV),
               k_weight=torch.from_numpy((1 + 0.3 * rng.standard_normal(128)).astype(np.float32)).to(DEV), interleaved=interleaved,
               kv_dtype=FLOAT[kind])
    want = cmc.cmc_norm_rope(q, k, v, pos, tf, **how)
    q[1, 2, 3, dim] = k[1, 2, 1, dim] = value
    got = cmc.cmc_norm_rope(q, k, v, pos, tf, **how)
    for y, w, at in ((got[0], want[0], (1, 2, 3)), (got[1], want[1], (1, 1, 2))):
        head = y[at]
        assert head.isnan().nonzero().flatten().tolist() == pair
        assert (head[~head.isnan()] == 0).all()
        y[at] = w[at]
        assert torch.equal(y, w)
    assert torch.equal(got[2], want[2])


def test_parts_left_out():
    rng = np.random.default_rng(7)
    q, k, v = projection(rng, 2, 3, 4, 2, 64, "bf16")
    f, tf = freqs(64)
    pos = torch.arange(6, dtype=torch.int32, device=DEV).view(2, 3)
    w = torch.rand(64, device=DEV)
    all_ = cmc.cmc_norm_rope(q, k, v, pos, tf, q_weight=w, k_weight=w)
    alone = cmc.cmc_norm_rope(q, None, None, pos, tf, q_weight=w)
    assert torch.equal(alone[0], all_[0]) and alone[1] is None and alone[2] is None
    keys = cmc.cmc_norm_rope(None, k, v, pos, tf, k_weight=w)
    assert keys[0] is None and torch.equal(keys[1], all_[1]) and torch.equal(keys[2], all_[2])
    keys = cmc.cmc_norm_rope(None, k, None, pos, tf, k_weight=w)
    assert keys[2] is None and torch.equal(keys[1], all_[1])
    only_q = cmc.cmc_norm_rope(q, k, v, pos, tf, q_weight=w)  # a norm for one of the two
    assert torch.equal(only_q[0], all_[0]) and not torch.equal(only_q[1], all_[1])


def test_empty():
    x = torch.empty(0, 3, 4, 64, device=DEV)
    q, k, v = cmc.cmc_norm_rope(x, x, x, torch.empty(0, 3, dtype=torch.int32, device=DEV), freqs(64)[1])
    assert q.shape == (0, 3, 4, 64) and k.shape == (0, 4, 3, 64)
    x = torch.empty(2, 0, 4, 64, device=DEV)
    assert cmc.cmc_norm_rope(x, None, None, torch.empty(2, 0, dtype=torch.int32, device=DEV), freqs(64)[1])[0].shape == x.shape


def test_separate_tensors_equal_slices():
    rng = np.random.default_rng(8)
    q, k, v = projection(rng, 3, 4, 8, 2, 128, "bf16")
    f, tf = freqs(128)
    pos = torch.arange(12, dtype=torch.int32, device=DEV).view(3, 4)
    a = cmc.cmc_norm_rope(q, k, v, pos, tf)
    b = cmc.cmc_norm_rope(q.contiguous(), k.contiguous(), v.contiguous(), pos, tf)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("Hq,Hkv,Dh,interleaved,kinds", [(5, 3, 64, False, ("bf16", "f32")), (48, 8, 64, False, ("bf16", "bf16")),
                                                        (48, 8, 64, True, ("f32", "bf16")), (90, 1, 256, False, ("f32", "f32"))])
def test_larger_launches_give_the_same_bits(Hq, Hkv, Dh, interleaved, kinds):
    """Outputs that pass the caches and such as do not; a token's heads in one workgroup
    and in several."""
    rng = np.random.default_rng(9)
    q, k, v = projection(rng, 1, 2050, Hq, Hkv, Dh, kinds[0])
    f, tf = freqs(48)
    pos = torch.arange(2050, dtype=torch.int32, device=DEV).view(1, 2050) * 7
    how = dict(q_weight=torch.rand(Dh, device=DEV), k_weight=torch.rand(Dh, device=DEV), interleaved=interleaved,
               q_dtype=FLOAT[kinds[1]], kv_dtype=torch.bfloat16)
    a = cmc.cmc_norm_rope(q, k, v, pos, tf, **how)
    for lo, hi in ((0, 900), (900, 2050)):
        b = cmc.cmc_norm_rope(q[:, lo:hi], k[:, lo:hi], v[:, lo:hi], pos[:, lo:hi].contiguous(), tf, **how)
        assert torch.equal(b[0], a[0][:, lo:hi]) and torch.equal(b[1], a[1][:, :, lo:hi]) and torch.equal(b[2], a[2][:, :, lo:hi])
    few = cmc.cmc_norm_rope(q[:, :, :3], k, None, pos, tf, **how)
    assert torch.equal(few[0], a[0][:, :, :3]) and torch.equal(few[1], a[1]) and few[2] is None


def test_more_threads_than_a_grid_dimension_holds():
    """2^26 + 5 tokens of one head: 2^32 threads and more, and offsets past 32 bits."""
    T = (1 << 26) + 5
    say("rope", T)
    q = torch.empty(1, T, 1, 64, dtype=torch.bfloat16, device=DEV)
    q.view(-1)[:64 * 1000].normal_()
    q[:, -1000:] = torch.randn(1, 1000, 1, 64, device=DEV).to(torch.bfloat16)
    pos = torch.arange(T, dtype=torch.int32, device=DEV).view(1, T)
    _, tf = freqs(64)
    got = cmc.cmc_norm_rope(q, None, None, pos, tf, q_dtype=torch.bfloat16)[0]
    for at in (slice(0, 1000), slice(T - 1000, T)):
        few = cmc.cmc_norm_rope(q[:, at], None, None, pos[:, at].contiguous(), tf, q_dtype=torch.bfloat16)[0]
        assert torch.equal(got[:, at], few)


# ------------------------------------------------------------- all together

def flow_inputs(seed, steps=3):
    rng = np.random.default_rng(seed)
    B, Hq, Hkv, Dh, N, k, W, P = 2, 8, 2, 128, 60, 20, 48, 70
    r = dict(B=B, Hq=Hq, Hkv=Hkv, Dh=Dh, N=N, k=k, W=W, P=P, steps=steps)
    r["mem"] = projection(rng, B, N, Hq, Hkv, Dh, "bf16")
    r["prompt"] = projection(rng, B, P, Hq, Hkv, Dh, "bf16")
    r["tokens"] = [projection(rng, B, 1, Hq, Hkv, Dh, "bf16") for _ in range(steps)]
    pos = lambda a, n: (torch.arange(a, a + n, dtype=torch.int32, device=DEV)[None] + torch.tensor([[0], [1000]], device=DEV)).to(
        torch.int32).contiguous()
    r["mem_pos"], r["prompt_pos"] = pos(0, N), pos(N, P)
    r["pos"] = [pos(N + P + t, 1) for t in range(steps)]
    r["f"] = freqs(128)[1]
    r["w"] = [torch.from_numpy((1 + 0.2 * rng.standard_normal(Dh)).astype(np.float32)).to(DEV) for _ in range(2)]
    r["idx"] = torch.from_numpy(np.stack([np.sort(rng.choice(N, k, replace=False)) for _ in range(B)]).astype(np.int32)).to(DEV)
    return r


def flow_state(r):
    u8 = lambda R, n: torch.zeros(r["B"], r["Hkv"], R, n, dtype=torch.uint8, device=DEV)
    Dh = r["Dh"]
    s = {x: [u8(R, Dh // 2), u8(R, Dh // 2), u8(R, Dh // 32), u8(R, Dh // 32)] for x, R in (("tier", r["k"]), ("ring", r["W"]))}
    s["count"] = torch.zeros(r["B"], dtype=torch.int32, device=DEV)
    s["out"] = [torch.zeros(r["B"], r["Hq"], Dh, device=DEV) for _ in range(r["steps"])]
    s["ws"] = cmc.decode_workspace_q4(r["B"], r["Hq"], r["Hkv"], Dh, r["k"], r["W"], DEV)
    new = lambda T: [torch.zeros(r["B"], r["Hkv"], T, Dh, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    s["pool"], s["prompt"], s["new"] = new(r["N"]), new(r["P"]), [new(1) for _ in range(r["steps"])]
    s["q"] = [torch.zeros(r["B"], 1, r["Hq"], Dh, device=DEV) for _ in range(r["steps"])]
    s["read"] = new(r["W"])
    return s


def flow_run(r, s):
    """Memory rows and a prompt into the cache, then some decode steps."""
    qw, kw = r["w"]
    rope = lambda x, pos, out, q=None: cmc.cmc_norm_rope(x[0] if q is not None else None, x[1], x[2], pos, r["f"], q_weight=qw,
                                                         k_weight=kw, out_q=q, out_k=out[0], out_v=out[1])
    s["count"].zero_()
    rope(r["mem"], r["mem_pos"], s["pool"])
    cmc.cmc_gather_tier1_q4(*s["pool"], r["idx"], r["k"], out_k=s["tier"][0], out_v=s["tier"][1], out_ks=s["tier"][2],
                            out_vs=s["tier"][3])
    rope(r["prompt"], r["prompt_pos"], s["prompt"])
    last = [x[:, :, -r["W"]:].contiguous() for x in s["prompt"]]
    cmc.cmc_window_append_q4(*s["ring"], s["count"], *last)
    for t in range(r["steps"]):
        rope(r["tokens"][t], r["pos"][t], s["new"][t], s["q"][t])
        cmc.cmc_decode_step_q4(s["q"][t].view(r["B"], r["Hq"], r["Dh"]), *s["tier"], r["k"], *s["ring"], s["count"], *s["new"][t],
                               r["Dh"] ** -0.5, out=s["out"][t], workspace=s["ws"])
    cmc.cmc_cache_read_q4(*s["ring"], count=s["count"], out_k=s["read"][0], out_v=s["read"][1])


def flow_outputs(s):
    return [*s["out"], *s["tier"], *s["ring"], s["count"], *s["read"], *s["pool"]]


def test_flow_together():
    """Each step's attention over the 4-bit values of the normed and rotated rows, and
    the rows' own distance from fp64 within their rounding."""
    r = flow_inputs(21)
    s = flow_state(r)
    flow_run(r, s)
    torch.cuda.synchronize()
    f = r["f"].cpu().numpy()
    w = [host(x) for x in r["w"]]
    for x, pos, got in ((r["mem"], r["mem_pos"], s["pool"]), (r["prompt"], r["prompt_pos"], s["prompt"])):
        want, bound = reference(host(x[1]), pos.cpu().numpy(), f, w[1], np.float32(1e-6), False)
        check(got[0], want.swapaxes(1, 2), bound.swapaxes(1, 2), "bf16")
    G = r["Hq"] // r["Hkv"]
    for b in range(r["B"]):
        for h in range(r["Hkv"]):
            lists = []
            for i in range(2):
                rows = np.concatenate([host(s["pool"][i])[b, h][r["idx"][b].cpu().numpy()], host(s["prompt"][i])[b, h][-r["W"]:],
                                       *[host(s["new"][t][i])[b, h] for t in range(r["steps"])]])
                lists.append(q4_ref.values(*q4_ref.quantise(rows)))
            for t in range(r["steps"]):
                keep = np.r_[0:r["k"], r["k"] + t + 1:r["k"] + r["W"] + t + 1]
                for g in range(G):
                    q, bound = reference(host(r["tokens"][t][0])[b:b + 1, :, h * G + g:h * G + g + 1], r["pos"][t][b:b + 1].cpu().numpy(), f,
                                         w[0], np.float32(1e-6), False)
                    assert (np.abs(host(s["q"][t])[b, 0, h * G + g] - q[0, 0, 0]) <= bound[0, 0, 0] + np.abs(q[0, 0, 0]) * 2.0 ** -23).all()
                    want, tol = q4_ref.attend(host(s["q"][t])[b, 0, h * G + g], lists[0][keep], lists[1][keep], r["Dh"] ** -0.5)
                    assert (np.abs(host(s["out"][t])[b, h * G + g] - want) <= tol).all()
            for i in range(2):
                assert (host(s["read"][i])[b, h] == lists[i][-r["W"]:]).all()
    assert s["count"].tolist() == [r["W"] + r["steps"]] * r["B"]


def test_flow_captured_and_replayed():
    r = flow_inputs(22)
    s, e = flow_state(r), flow_state(r)
    flow_run(r, s)  # first calls outside capture
    torch.cuda.synchronize()
    say("q4 flow: capturing")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        flow_run(r, s)
    for i in range(4):
        say("q4 flow: replay", i)
        for x in r["tokens"]:
            for t in x:
                t.mul_(0.9)
        g.replay()
        flow_run(r, e)
        torch.cuda.synchronize()
        for x, y in zip(flow_outputs(s), flow_outputs(e)):
            assert torch.equal(x, y), i
        a = torch.randn(256, 256, device=DEV)
        (a @ a).sum().item()


def test_two_streams_with_their_own_workspaces():
    r1, r2 = flow_inputs(23), flow_inputs(24)
    want = []
    for r in (r1, r2):
        s = flow_state(r)
        flow_run(r, s)
        want.append([t.clone() for t in flow_outputs(s)])
    s1, s2 = flow_state(r1), flow_state(r2)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        for st, r, s in zip(streams, (r1, r2), (s1, s2)):
            with torch.cuda.stream(st):
                flow_run(r, s)
    torch.cuda.synchronize()
    for s, w in ((s1, want[0]), (s2, want[1])):
        for x, y in zip(flow_outputs(s), w):
            assert torch.equal(x, y)


def test_on_a_side_stream_that_is_not_current():
    """Outputs and workspaces that the calls make themselves are theirs on that stream."""
    r = flow_inputs(25)
    s = flow_state(r)
    flow_run(r, s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy = torch.randn(2048, 2048, device=DEV)
    for _ in range(10):
        busy = (busy @ busy).clamp(-1, 1)
    q, k, v = cmc.cmc_norm_rope(*r["tokens"][0], r["pos"][0], r["f"], q_weight=r["w"][0], k_weight=r["w"][1], stream=side)
    out = cmc.cmc_two_tier_decode_q4(s["q"][2].view(r["B"], r["Hq"], r["Dh"]), *s["tier"], r["k"], *s["ring"], s["count"], r["Dh"] ** -0.5,
                                     stream=side)
    side.synchronize()
    assert torch.equal(q, s["q"][0]) and torch.equal(k, s["new"][0][0]) and torch.equal(v, s["new"][0][1])
    assert (out - s["out"][2]).abs().max() <= 1e-5  # the last step's attention, without its append in the launch
