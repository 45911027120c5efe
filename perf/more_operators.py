"""Performance cases of the 4-bit two-tier cache, and of the norms and the position
rotation that the rows go through before they reach any cache.

A 4-bit cache array (Tier-1 block or Tier-2 ring, K or V) is held as e2m1 codes,
two to a byte with the even dim in the low half, ``uint8 [B][Hkv][R][Dh / 2]``, and
one e8m0 scale for every 32 dims of a row, ``uint8 [B][Hkv][R][Dh / 32]``: a code's
sign, two exponent bits and one fraction bit stand for +-{0, .5, 1, 1.5, 2, 3, 4, 6},
a scale byte s for 2^(s - 127).  With a the largest finite magnitude of the 32
elements, s is the least byte >= 1 with a <= 6 * 2^(s - 127), and a code is its
element over the scale rounded to nearest even.

Kinds of work:

  step    one decode step of one layer: the step's rows appended to the ring, then
          attention over [Tier-1 rows || ring] (``cmc_decode_step_q4``); the ring's
          new rows are read back (``cmc_cache_read_q4``)
  attend  the attention alone (``cmc_two_tier_decode_q4``)
  tier1   once per question: the selected rows gathered and quantised
          (``cmc_gather_tier1_q4``), and read back
  append  rows written into the ring (``cmc_window_append_q4``), and read back
  rope    the heads of a projection normed and rotated, and laid out as the decode
          and the append take them (``cmc_norm_rope``)

``run`` computes them with elementary torch operations, or, where ``own`` is set, by
the calls above.
"""
import math

import torch

own = False

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
_FLOAT = {"bf16": BF16, "f32": F32}
_BYTES = {"bf16": 2, "f32": 4}
GROUP = 32


def listed():
    return [
        # One Llama-shaped layer at batch 1, 256 rows kept of a compressed
        # context and a window of 512: the latency of a single user's token.
        dict(name="step_b1", kind="step", B=1, Hq=32, Hkv=8, Dh=128, k=256, W=512, T=1, kv="bf16", ragged=False),
        # One Mistral-shaped layer for 64 sequences, every cache full: the
        # steady state of a batch server.
        dict(name="step_b64", kind="step", B=64, Hq=32, Hkv=8, Dh=128, k=512, W=1024, T=1, kv="bf16", ragged=False),
        # A mixed batch: per-sequence row counts, rings partly filled, odd
        # sizes, eight query heads to a kv head, several rows a step.
        dict(name="step_ragged_g8", kind="step", B=24, Hq=64, Hkv=8, Dh=128, k=549, W=1000, T=4, kv="f32", ragged=True),
        # Wide heads without query grouping over a long window.
        dict(name="attend_wide", kind="attend", B=16, Hq=16, Hkv=16, Dh=256, k=1000, W=2048, T=0, kv="bf16", ragged=False),
        # One user's uncompressed cache: the whole context in the ring.
        dict(name="attend_long", kind="attend", B=1, Hq=32, Hkv=8, Dh=128, k=40, W=32768, T=0, kv="bf16", ragged=False),
        # One user's question: 256 of 2048 memory rows.
        dict(name="tier1_b1", kind="tier1", B=1, Hkv=8, Dh=128, N=2048, k=256, kv="bf16", ragged=False),
        # The questions of a mixed batch.
        dict(name="tier1_b64", kind="tier1", B=64, Hkv=8, Dh=128, N=4096, k=560, kv="f32", ragged=True),
        # A decode step's rows of 64 sequences, where the append is not fused.
        dict(name="append_b64", kind="append", B=64, Hkv=8, Dh=128, W=1024, T=1, kv="bf16"),
        # The local windows of 8 sequences written into their rings at prefill.
        dict(name="append_prefill", kind="append", B=8, Hkv=8, Dh=128, W=1024, T=1024, kv="bf16"),
        # One user's token: the heads of one projection row.
        dict(name="rope_b1", kind="rope", B=1, T=1, Hq=32, Hkv=8, Dh=128, rot=128, norm=True, pairs=False, kv="bf16", to="bf16"),
        # A step of 64 sequences with half of each head rotated, in neighbouring
        # pairs, eight query heads to a kv head.
        dict(name="rope_b64", kind="rope", B=64, T=1, Hq=64, Hkv=8, Dh=128, rot=64, norm=True, pairs=True, kv="f32", to="bf16"),
        # The prompts of two sequences at prefill.
        dict(name="rope_prefill", kind="rope", B=2, T=4096, Hq=32, Hkv=8, Dh=128, rot=128, norm=True, pairs=False, kv="bf16",
             to="bf16"),
    ]


# ------------------------------------------------------------------- draws

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the ranges above: batches of 1 to 64, every head shape and input
    type, lists of a few rows to 32768, prompts of one token to 8192; no more work
    than the largest listed case of its kind."""
    kind = rng.choice(["step", "step", "attend", "attend", "tier1", "append", "rope", "rope"])
    c = dict(kind=kind, B=_log_int(rng, 1, 64), kv=rng.choice(["bf16", "bf16", "f32"]), Dh=rng.choice([64, 128, 128, 256]))
    if kind in ("step", "attend", "rope"):
        c["Hq"], c["Hkv"] = rng.choice([(32, 8), (32, 8), (16, 16), (64, 8), (32, 16), (4, 4), (28, 7)])
    if kind in ("step", "attend"):
        c["k"] = _log_int(rng, 1, 2048)
        c["W"] = _log_int(rng, 16, 32768 if c["B"] < 8 else 4096)
        c["T"] = rng.choice([1, 1, 1, 4]) if kind == "step" else 0
        c["ragged"] = rng.random() < 0.4
        most = 1.1e8
    elif kind == "rope":
        c["T"] = rng.choice([1, 1, _log_int(rng, 1, 8192)])
        c["rot"] = rng.choice([c["Dh"], c["Dh"], c["Dh"] // 2, 16, 48])
        c["norm"] = rng.random() < 0.75
        c["pairs"] = rng.random() < 0.4
        c["to"] = rng.choice(["bf16", "bf16", "f32"])
        most = 2.6e8
    else:
        c["Hkv"] = rng.choice([4, 7, 8, 16])
        if kind == "tier1":
            c["N"] = _log_int(rng, 64, 8192)
            c["k"] = max(1, min(1024, c["N"] // rng.choice([2, 4, 8])))
            c["ragged"] = rng.random() < 0.5
            most = 2.5e8
        else:
            c["W"] = _log_int(rng, 16, 8192)
            c["T"] = rng.choice([1, 1, _log_int(rng, 1, c["W"]), c["W"]])
            most = 9e7
    while work(c)["bytes"] > most:
        if c["B"] > 1:
            c["B"] = (c["B"] + 1) // 2
        elif kind == "append":
            c["W"], c["T"] = (c["W"] + 1) // 2, (c["T"] + 1) // 2
        else:
            c["T" if kind == "rope" else "W" if kind in ("step", "attend") else "k"] //= 2
    while "N" in c and c["N"] > c["k"] and c["B"] * c["Hkv"] * c["N"] * c["Dh"] * _BYTES[c["kv"]] > 1.1e9:
        c["N"] = max(c["k"], c["N"] // 2)
    return c


# ------------------------------------------------------------- plain forms

def _quantise(x):
    """x [..][Dh] fp32 -> codes uint8 [..][Dh / 2], scale bytes uint8 [..][Dh / 32]."""
    g = x.unflatten(-1, (-1, GROUP))
    a = torch.where(g.isfinite(), g.abs(), torch.zeros((), device=x.device)).amax(dim=-1)
    m, e = torch.frexp(a)  # a = m 2^e, m in [1/2, 1); 6 = 3/4 * 2^3
    byte = torch.where(a > 0, e - 3 + (m > 0.75) + 127, 1).clamp(min=1).to(torch.int32)
    y = (g.abs() / (byte << 23).view(F32)[..., None]).clamp(max=6.0)
    code = torch.where(y < 2, (2 * y).round(), torch.where(y < 4, 2 + y.round(), 4 + (y / 2).round()))
    code = code.to(torch.uint8) + 8 * g.signbit().to(torch.uint8)
    nan = g.isnan().any(dim=-1)  # which its whole group then is
    code = torch.where(nan[..., None], torch.zeros_like(code), code).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], torch.where(nan, 255, byte).to(torch.uint8)


def _values(codes, scales):
    """fp32 values [..][Dh]; a row that was never written may give anything."""
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    mag = (c & 7).to(F32)
    v = torch.where(mag < 4, mag / 2, torch.where(mag < 6, mag - 2, 2 * mag - 8))
    v = torch.where(c >= 8, -v, v).unflatten(-1, (-1, GROUP))
    return (v * (scales.to(torch.int32) << 23).view(F32)[..., None]).flatten(-2)


def _live_values(codes, scales, live):
    v = _values(codes, scales)
    return torch.where(live[..., None], v, torch.zeros((), device=v.device))


def _count_mask(count, R):
    """[B][1][R]: the rows below each sequence's count."""
    return (torch.arange(R, device=count.device)[None, :] < count[:, None])[:, None]


def _plain_append(s):
    """The ring after this call's rows, in the state's own buffers."""
    W, T, count = s["win_k"].shape[2], s["new_k"].shape[2], s["win_count"]
    slot = ((count[:, None] + torch.arange(T, device=DEV)[None, :]) % W)[:, None, :, None]
    for x in ("k", "v"):
        for to, what in zip(("win_" + x, "win_" + x + "s"), _quantise(s["new_" + x].to(F32))):
            s[to].scatter_(2, slot.expand(-1, what.shape[1], -1, what.shape[3]), what)
    count += T


def _plain_read(s, codes, scales, count, rows):
    """The newest `rows` rows of an array into the state's rows_k/v, oldest first."""
    R = s[codes + "k"].shape[2]
    count = torch.full((s[codes + "k"].shape[0],), R, device=DEV) if count is None else count
    n = count.clamp(max=R)
    m = n.clamp(max=rows)
    at = ((count - m)[:, None] + torch.arange(rows, device=DEV)[None, :]) % R
    live = _count_mask(m, rows)
    for x in ("k", "v"):
        put = [s[a].gather(2, at[:, None, :, None].expand(-1, s[a].shape[1], -1, s[a].shape[3]))
               for a in (codes + x, scales % x)]
        s["rows_" + x].copy_(torch.where(live[..., None], _values(*put).to(s["rows_" + x].dtype), s["rows_" + x]))


def _plain_attend(s):
    B, Hq, Dh = s["q"].shape
    Hkv = s["win_k"].shape[1]
    k_len = s["k_len"] if s["k_len"] is not None else torch.full((B,), s["k"], device=DEV)
    lives = _count_mask(k_len, s["k"]), _count_mask(s["win_count"], s["win_k"].shape[2])
    live = torch.cat(lives, dim=2)
    K, V = (torch.cat([_live_values(s["cme_" + x], s["cme_" + x + "s"], lives[0]),
                       _live_values(s["win_" + x], s["win_" + x + "s"], lives[1])], dim=2) for x in ("k", "v"))
    q = s["q"].view(B, Hkv, Hq // Hkv, Dh) * s["scale"]
    z = (q @ K.transpose(2, 3)).masked_fill(~live[:, :, None], -math.inf)
    top = z.amax(dim=3, keepdim=True)
    p = torch.exp(z - torch.where(top.isinf(), torch.zeros_like(top), top))
    den = p.sum(dim=3, keepdim=True)
    return ((p @ V) / torch.where(den > 0, den, torch.ones_like(den))).view(B, Hq, Dh)


def _plain_rotate(x, angle, weight, eps, pairs):
    """x [B][T][H][Dh] fp32 normed and rotated by angle [B][T][rot / 2] (fp64)."""
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + eps) * weight
    half = angle.shape[-1]
    cos, sin = (f(angle).to(F32)[:, :, None, :] for f in (torch.cos, torch.sin))
    r, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (r[..., 0::2], r[..., 1::2]) if pairs else (r[..., :half], r[..., half:])
    turned = [a * cos - b * sin, b * cos + a * sin]
    r = torch.stack(turned, dim=-1).flatten(-2) if pairs else torch.cat(turned, dim=-1)
    return torch.cat([r, rest], dim=-1)


# ------------------------------------------------------------------ inputs

class _Draws:
    """Seeded draws on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device=DEV, dtype=F32)

    def ints(self, lo, hi, *shape):
        return torch.randint(lo, hi + 1, shape, generator=self.g, device=DEV, dtype=torch.int32)

    def rows(self, shape, kv, spread):
        """K or V rows of one type: N(0, 1), with channels of different sizes
        (keys more than values) as decoders have them."""
        B, H, R, D = shape
        x = self.normal(*shape)
        x *= torch.exp(spread * self.normal(1, H, 1, D))
        return x.to(_FLOAT[kv])


_SPREAD = (("k", 0.7), ("v", 0.3))


def _prepare_ring(c, d, count):
    """A 4-bit ring filled up to min(count, W)."""
    s = dict(win_count=count)
    live = _count_mask(count, c["W"])[..., None]
    for x, spread in _SPREAD:
        rows = d.rows((c["B"], c["Hkv"], c["W"], c["Dh"]), c["kv"], spread).to(F32)
        s["win_" + x], s["win_" + x + "s"] = _quantise(torch.where(live, rows, torch.zeros((), device=DEV)))
    return s


def _rows_out(s, shape):
    for x in ("k", "v"):
        s["rows_" + x] = torch.zeros(shape, dtype=BF16, device=DEV)  # which holds every value of the cache


def _prepare_decode(c, seed):
    d = _Draws(seed)
    B, Hq, Hkv, Dh, k, W = (c[x] for x in ("B", "Hq", "Hkv", "Dh", "k", "W"))
    if c["ragged"]:  # from a quarter of the rows up, rings from a quarter full to wrapped
        k_len, count = d.ints(max(1, k // 4), k, B), d.ints(max(1, W // 4), 2 * W, B)
    else:
        k_len, count = None, torch.full((B,), W + 3, dtype=torch.int32, device=DEV)
    s = _prepare_ring(c, d, count)
    for x, spread in _SPREAD:
        s["cme_" + x], s["cme_" + x + "s"] = _quantise(d.rows((B, Hkv, k, Dh), c["kv"], spread).to(F32))
        if c["T"]:
            s["new_" + x] = d.rows((B, Hkv, c["T"], Dh), c["kv"], spread)
    if c["T"]:
        _rows_out(s, (B, Hkv, c["T"], Dh))
    s.update(k=k, k_len=k_len, q=d.normal(B, Hq, Dh), scale=1.0 / math.sqrt(Dh),
             out=torch.empty((B, Hq, Dh), dtype=F32, device=DEV))
    return s


_prepare_step = _prepare_attend = _prepare_decode


def _prepare_tier1(c, seed):
    d = _Draws(seed)
    B, Hkv, Dh, N, k = (c[x] for x in ("B", "Hkv", "Dh", "N", "k"))
    idx = torch.rand((B, N), generator=d.g, device=DEV).topk(k, dim=1).indices.sort(dim=1).values.to(torch.int32)
    s = dict(k=k, idx=idx.contiguous(), k_len=d.ints(max(1, k // 4), k, B) if c["ragged"] else None)
    for x, spread in _SPREAD:
        s["cme_" + x] = d.rows((B, Hkv, N, Dh), c["kv"], spread)
        # rows past a sequence's count stay as they are
        s["out_" + x] = torch.zeros((B, Hkv, k, Dh // 2), dtype=torch.uint8, device=DEV)
        s["out_" + x + "s"] = torch.zeros((B, Hkv, k, Dh // GROUP), dtype=torch.uint8, device=DEV)
    _rows_out(s, (B, Hkv, k, Dh))
    return s


def _prepare_append(c, seed):
    d = _Draws(seed)
    B, Hkv, Dh, W, T = (c[x] for x in ("B", "Hkv", "Dh", "W", "T"))
    # a prefill starts an empty ring, a step finds one in use
    count = torch.zeros((B,), dtype=torch.int32, device=DEV) if T == W else d.ints(W // 2, 3 * W, B)
    s = _prepare_ring(c, d, count)
    for x, spread in _SPREAD:
        s["new_" + x] = d.rows((B, Hkv, T, Dh), c["kv"], spread)
    _rows_out(s, (B, Hkv, T, Dh))
    return s


def _prepare_rope(c, seed):
    d = _Draws(seed)
    B, T, Hq, Hkv, Dh, rot = (c[x] for x in ("B", "T", "Hq", "Hkv", "Dh", "rot"))
    # one projection's output, a token's heads of q, k and v side by side
    x = d.normal(B, T, (Hq + 2 * Hkv), Dh)
    x *= torch.exp(0.5 * d.normal(1, 1, Hq + 2 * Hkv, Dh))
    x = x.to(_FLOAT[c["kv"]])
    s = dict(x=x, q=x[:, :, :Hq], k=x[:, :, Hq:Hq + Hkv], v=x[:, :, Hq + Hkv:], pairs=c["pairs"], eps=1e-6)
    start = d.ints(0, 1 << 17, B, 1)
    s["pos"] = (start + torch.arange(T, device=DEV, dtype=torch.int32)[None, :]).contiguous()
    s["inv_freq"] = (500000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)).to(F32)
    for h in ("q", "k"):
        s[h + "_weight"] = 1.0 + 0.2 * d.normal(Dh) if c["norm"] else None
    to = _FLOAT[c["to"]]
    s["out_q"] = torch.empty((B, T, Hq, Dh), dtype=F32, device=DEV)
    s["out_k"], s["out_v"] = (torch.empty((B, Hkv, T, Dh), dtype=to, device=DEV) for _ in range(2))
    return s


def prepare(case, seed):
    return dict(kind=case["kind"], **globals()["_prepare_" + case["kind"]](case, seed))


# -------------------------------------------------------------------- runs

def _workspace(s):
    """The decode workspace, made at the first pass and kept, as a serving
    program keeps it."""
    from paper_2609_25537_amd import cmc
    if "workspace" not in s:
        B, Hq, Dh = s["q"].shape
        s["workspace"] = cmc.decode_workspace_q4(B, Hq, s["win_k"].shape[1], Dh, s["k"], s["win_k"].shape[2], DEV)
    return s["workspace"]


def _run_step(s):
    if own:
        from paper_2609_25537_amd import cmc
        cmc.cmc_decode_step_q4(s["q"], s["cme_k"], s["cme_v"], s["cme_ks"], s["cme_vs"], s["k"], s["win_k"], s["win_v"],
                               s["win_ks"], s["win_vs"], s["win_count"], s["new_k"], s["new_v"], s["scale"],
                               k_len=s["k_len"], out=s["out"], workspace=_workspace(s))
        cmc.cmc_cache_read_q4(s["win_k"], s["win_v"], s["win_ks"], s["win_vs"], count=s["win_count"], out_k=s["rows_k"],
                              out_v=s["rows_v"])
        out = s["out"]
    else:
        _plain_append(s)
        out = _plain_attend(s)
        _plain_read(s, "win_", "win_%ss", s["win_count"], s["new_k"].shape[2])
    return dict(out=out, **{x: s[x] for x in ("rows_k", "rows_v", "win_count")})


def _run_attend(s):
    if own:
        from paper_2609_25537_amd import cmc
        return cmc.cmc_two_tier_decode_q4(s["q"], s["cme_k"], s["cme_v"], s["cme_ks"], s["cme_vs"], s["k"], s["win_k"],
                                          s["win_v"], s["win_ks"], s["win_vs"], s["win_count"], s["scale"],
                                          k_len=s["k_len"], out=s["out"], workspace=_workspace(s))
    return _plain_attend(s)


def _run_tier1(s):
    if own:
        from paper_2609_25537_amd import cmc
        out = [s[x] for x in ("out_k", "out_v", "out_ks", "out_vs")]
        cmc.cmc_gather_tier1_q4(s["cme_k"], s["cme_v"], s["idx"], s["k"], k_len=s["k_len"], out_k=out[0], out_v=out[1],
                                out_ks=out[2], out_vs=out[3])
        cmc.cmc_cache_read_q4(*out, count=s["k_len"], out_k=s["rows_k"], out_v=s["rows_v"])
    else:
        B, k = s["idx"].shape
        live = _count_mask(s["k_len"] if s["k_len"] is not None else torch.full((B,), k, device=DEV), k)[..., None]
        for x in ("k", "v"):
            pool = s["cme_" + x]
            at = s["idx"].long()[:, None, :, None].expand(-1, pool.shape[1], -1, pool.shape[3])
            for to, what in zip(("out_" + x, "out_" + x + "s"), _quantise(pool.gather(2, at).to(F32))):
                s[to].copy_(torch.where(live, what, s[to]))
        _plain_read(s, "out_", "out_%ss", s["k_len"], k)
    return {x: s[x] for x in ("rows_k", "rows_v")}


def _run_append(s):
    if own:
        from paper_2609_25537_amd import cmc
        cmc.cmc_window_append_q4(s["win_k"], s["win_v"], s["win_ks"], s["win_vs"], s["win_count"], s["new_k"], s["new_v"])
        cmc.cmc_cache_read_q4(s["win_k"], s["win_v"], s["win_ks"], s["win_vs"], count=s["win_count"], out_k=s["rows_k"],
                              out_v=s["rows_v"])
    else:
        _plain_append(s)
        _plain_read(s, "win_", "win_%ss", s["win_count"], s["new_k"].shape[2])
    return {x: s[x] for x in ("rows_k", "rows_v", "win_count")}


def _run_rope(s):
    out = {x: s[x] for x in ("out_q", "out_k", "out_v")}
    if own:
        from paper_2609_25537_amd import cmc
        cmc.cmc_norm_rope(s["q"], s["k"], s["v"], s["pos"], s["inv_freq"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                          eps=s["eps"], interleaved=s["pairs"], **out)
        return out
    angle = s["pos"].double()[..., None] * s["inv_freq"].double()
    out["out_q"].copy_(_plain_rotate(s["q"].to(F32), angle, s["q_weight"], s["eps"], s["pairs"]))
    out["out_k"].copy_(_plain_rotate(s["k"].to(F32), angle, s["k_weight"], s["eps"], s["pairs"]).transpose(1, 2))
    out["out_v"].copy_(s["v"].transpose(1, 2))
    return out


def run(state):
    return globals()["_run_" + state["kind"]](state)


# -------------------------------------------------------------------- work

def work(case):
    """What a pass cannot do without: every live code, scale and input read
    once, every output written once.  Ragged counts enter with their means."""
    c = case
    B, Hkv, Dh = c["B"], c["Hkv"], c["Dh"]
    row = 2 * Hkv * Dh  # elements of a row, K and V
    code = 0.5 + 1.0 / GROUP  # bytes of an element
    ragged = c.get("ragged", False)
    if c["kind"] in ("step", "attend"):
        # the ring's share: mean of min(count, W) / W for counts from W / 4 to 2 W
        keys = c["k"] * (0.625 if ragged else 1.0) + c["W"] * (0.8571 if ragged else 1.0)
        wrote = c["T"] * (_BYTES[c["kv"]] + code + 2)
        return {"bytes": B * (row * (keys * code + wrote) + 8 * c["Hq"] * Dh), "flops": 4.0 * B * c["Hq"] * keys * Dh}
    if c["kind"] == "tier1":
        keys = c["k"] * (0.625 if ragged else 1.0)
        return {"bytes": B * (row * keys * (_BYTES[c["kv"]] + 2 * code + 2) + 4 * keys), "flops": 3.0 * B * row * keys}
    if c["kind"] == "append":
        return {"bytes": B * row * c["T"] * (_BYTES[c["kv"]] + 2 * code + 2.0), "flops": 3.0 * B * row * c["T"]}
    token = (c["Hq"] + 2 * Hkv) * Dh * _BYTES[c["kv"]] + c["Hq"] * Dh * 4 + row * _BYTES[c["to"]] + 4
    return {"bytes": B * c["T"] * token, "flops": 7.0 * B * c["T"] * (c["Hq"] + Hkv) * Dh}


# ------------------------------------------------------------------- exact

_TABLE = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_quantised(x):
    """The values that rows (fp64, [..][Dh]) stand for in 4 bits, from the definition:
    the least power of two, then the nearest of the eight magnitudes, of two the one
    with the even code."""
    g = x.unflatten(-1, (-1, GROUP))
    a = g.abs().amax(dim=-1, keepdim=True)
    s = torch.full_like(a, 2.0 ** -126)
    e = torch.floor(torch.log2((a / 6).clamp(min=2.0 ** -126))) - 1  # log2 may be off by a rounding: count up from below
    s = torch.maximum(s, torch.exp2(e))
    for _ in range(3):
        s = torch.where(a > 6 * s, 2 * s, s)
    y, r = g.abs() / s, torch.zeros_like(g)
    for i in range(1, 8):
        mid = (_TABLE[i - 1] + _TABLE[i]) / 2
        r = torch.where(y >= mid if i % 2 == 0 else y > mid, torch.full_like(r, _TABLE[i]), r)
    return (torch.copysign(r, g) * s).flatten(-2)


def _exact_values(codes, scales):
    table = torch.tensor(_TABLE + tuple(-v for v in _TABLE), dtype=torch.float64, device=DEV)
    lo, hi = table[(codes % 16).long()], table[(codes // 16).long()]
    v = torch.stack([lo, hi], dim=-1).flatten(-2)
    return v * torch.exp2(scales.double() - 127).repeat_interleave(GROUP, dim=-1)


def _exact_ring(s):
    """Each sequence's ring after the append: values [B][Hkv][W][Dh] in fp64."""
    r = {x: _exact_values(s["win_" + x], s["win_" + x + "s"]) for x in ("k", "v")}
    if "new_k" in s:
        W, T = s["win_k"].shape[2], s["new_k"].shape[2]
        new = {x: _exact_quantised(s["new_" + x].double()) for x in ("k", "v")}
        for b, count in enumerate(s["win_count"].tolist()):
            slots = (count + torch.arange(T, device=DEV)) % W
            for x in ("k", "v"):
                r[x][b][:, slots] = new[x][b]
    return r


def _exact_attend(s, ring, counts):
    """Each sequence's attention over its own list of keys, in fp64."""
    B, Hq, Dh = s["q"].shape
    Hkv, W = s["win_k"].shape[1], s["win_k"].shape[2]
    out = torch.zeros((B, Hkv, Hq // Hkv, Dh), dtype=torch.float64, device=DEV)
    for b in range(B):
        n, w = s["k"] if s["k_len"] is None else int(s["k_len"][b]), min(int(counts[b]), W)
        K, V = (torch.cat([_exact_values(s["cme_" + x][b, :, :n], s["cme_" + x + "s"][b, :, :n]), ring[x][b, :, :w]], dim=1)
                for x in ("k", "v"))
        q = s["q"][b].double().view(Hkv, Hq // Hkv, Dh)
        out[b] = torch.softmax(torch.matmul(q, K.transpose(1, 2).contiguous()) / math.sqrt(Dh), dim=2) @ V
    return out.view(B, Hq, Dh)


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind in ("step", "append"):
        count, new = s["win_count"].long() + case["T"], {"rows_" + x: _exact_quantised(s["new_" + x].double()) for x in ("k", "v")}
        r = dict(win_count=count, **new)
        return dict(out=_exact_attend(s, _exact_ring(s), count), **r) if kind == "step" else r
    if kind == "attend":
        return _exact_attend(s, _exact_ring(s), s["win_count"])
    if kind == "tier1":
        r = {x: s[x].double() for x in ("rows_k", "rows_v")}
        for b in range(case["B"]):
            n = s["k"] if s["k_len"] is None else int(s["k_len"][b])
            for x in ("k", "v"):
                r["rows_" + x][b, :, :n] = _exact_quantised(s["cme_" + x][b][:, s["idx"][b, :n].long()].double())
        return r
    angle = s["pos"].double()[..., None] * s["inv_freq"].double()
    turn = torch.polar(torch.ones_like(angle), angle)[:, :, None]
    out = {}
    for h in ("q", "k"):
        x = s[h].double()
        if case["norm"]:
            x = x / torch.sqrt((x * x).sum(dim=-1, keepdim=True) / case["Dh"] + s["eps"]) * s[h + "_weight"].double()
        r = x[..., :case["rot"]]
        if case["pairs"]:
            z = torch.view_as_complex(r.unflatten(-1, (-1, 2)).contiguous()) * turn
            r = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(*(y.contiguous() for y in r.chunk(2, dim=-1))) * turn
            r = torch.cat([z.real, z.imag], dim=-1)
        out["out_" + h] = torch.cat([r, x[..., case["rot"]:]], dim=-1)
    return dict(out_q=out["out_q"], out_k=out["out_k"].transpose(1, 2), out_v=s["v"].double().transpose(1, 2))
