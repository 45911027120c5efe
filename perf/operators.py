"""Performance cases of the 8-bit two-tier cache: writing it, reading it back, and
the decode attention over it.

A cache array (Tier-1 block or Tier-2 ring, K or V) is held as 8-bit codes
``[B][Hkv][R][Dh]`` (``float8_e4m3fn`` or ``int8``) with one fp32 scale for each
block of ``block`` rows of a head, ``[B][Hkv][ceil(R / block)]``; a row's value
is code times scale.  With a the largest finite magnitude of a block's live
rows and M the codes' largest (448, 127), the scale is the least power of two s
>= 2^-126 with a <= M s, and the code is x / s rounded to nearest even.

Kinds of work:

  step    one decode step of one layer: the step's rows appended to the ring,
          then attention over [Tier-1 rows || ring] (``cmc_decode_step_q8``)
  attend  the attention alone (``cmc_two_tier_decode_q8``)
  tier1   once per question: the selected rows gathered and quantised
          (``cmc_gather_tier1_q8``)
  append  rows written into the ring (``cmc_window_append_q8``)
  read    the ring read back, oldest row first (``cmc_cache_read_q8``)

``run`` computes them with elementary torch operations, or, where ``own`` is
set, by the calls above.
"""
import math

import torch

own = False

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
E4M3, I8 = torch.float8_e4m3fn, torch.int8
_CODE = {"e4m3": E4M3, "i8": I8}
_FLOAT = {"bf16": BF16, "f32": F32}
_BYTES = {"bf16": 2, "f32": 4}
_MOST = {E4M3: 448.0, I8: 127.0}


def listed():
    return [
        # One Llama-shaped layer at batch 1, 256 rows kept of a compressed
        # context and a window of 512: the latency of a single user's token.
        dict(name="step_b1", kind="step", B=1, Hq=32, Hkv=8, Dh=128, k=256, W=512, T=1, code="e4m3", block=32, kv="bf16",
             ragged=False),
        # One Mistral-shaped layer for 64 sequences, every cache full: the
        # steady state of a batch server.
        dict(name="step_b64", kind="step", B=64, Hq=32, Hkv=8, Dh=128, k=512, W=1024, T=1, code="e4m3", block=32,
             kv="bf16", ragged=False),
        # A mixed batch: per-sequence row counts, rings partly filled, odd
        # sizes, eight query heads to a kv head, several rows a step.
        dict(name="step_ragged_g8", kind="step", B=24, Hq=64, Hkv=8, Dh=128, k=549, W=1000, T=4, code="i8", block=64,
             kv="f32", ragged=True),
        # Wide heads without query grouping over a long window.
        dict(name="attend_wide", kind="attend", B=16, Hq=16, Hkv=16, Dh=256, k=1024, W=2048, T=0, code="e4m3", block=128,
             kv="bf16", ragged=False),
        # One user's uncompressed cache: the whole context in the ring.
        dict(name="attend_long", kind="attend", B=1, Hq=32, Hkv=8, Dh=128, k=40, W=32768, T=0, code="i8", block=32,
             kv="bf16", ragged=False),
        # Small heads in pairs, a few sequences of different lengths.
        dict(name="attend_small", kind="attend", B=8, Hq=16, Hkv=8, Dh=64, k=200, W=500, T=0, code="e4m3", block=32,
             kv="bf16", ragged=True),
        # One user's question: 256 of 2048 memory rows.
        dict(name="tier1_b1", kind="tier1", B=1, Hkv=8, Dh=128, N=2048, k=256, code="e4m3", block=32, kv="bf16",
             ragged=False),
        # The questions of a mixed batch.
        dict(name="tier1_b64", kind="tier1", B=64, Hkv=8, Dh=128, N=4096, k=560, code="i8", block=64, kv="f32",
             ragged=True),
        # A decode step's rows of 64 sequences, where the append is not fused.
        dict(name="append_b64", kind="append", B=64, Hkv=8, Dh=128, W=1024, T=1, code="e4m3", block=32, kv="bf16"),
        # The local windows of 8 sequences written into their rings at prefill.
        dict(name="append_prefill", kind="append", B=8, Hkv=8, Dh=128, W=1024, T=1024, code="e4m3", block=32, kv="bf16"),
        # A small window read back.
        dict(name="read_b1", kind="read", B=1, Hkv=8, Dh=128, W=512, code="e4m3", block=32, kv="bf16", ragged=False),
        # The windows of a mixed batch.
        dict(name="read_b64", kind="read", B=64, Hkv=8, Dh=128, W=1000, code="i8", block=64, kv="bf16", ragged=True),
    ]


# ------------------------------------------------------------------- draws

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the ranges above: batches of 1 to 64, every head shape, code,
    block and input type, lists of a few rows to 32768; no more work than the
    largest listed case of its kind."""
    kind = rng.choice(["step", "step", "attend", "attend", "tier1", "append", "read"])
    c = dict(kind=kind, B=_log_int(rng, 1, 64), code=rng.choice(["e4m3", "i8"]), block=rng.choice([32, 32, 64, 128]),
             kv=rng.choice(["bf16", "bf16", "f32"]), Dh=rng.choice([64, 128, 128, 256]))
    if kind in ("step", "attend"):
        c["Hq"], c["Hkv"] = rng.choice([(32, 8), (32, 8), (16, 16), (64, 8), (32, 16), (4, 4), (28, 7)])
        c["k"] = _log_int(rng, 1, 2048)
        c["W"] = _log_int(rng, 16, 32768 if c["B"] < 8 else 4096)
        c["T"] = rng.choice([1, 1, 1, 4]) if kind == "step" else 0
        c["ragged"] = rng.random() < 0.4
        most = 2.2e8
    else:
        c["Hkv"] = rng.choice([4, 7, 8, 16])
        if kind == "tier1":
            c["N"] = _log_int(rng, 64, 8192)
            c["k"] = max(1, min(1024, c["N"] // rng.choice([2, 4, 8])))
            c["ragged"] = rng.random() < 0.5
        else:
            c["W"] = _log_int(rng, 16, 8192)
        if kind == "append":
            c["T"] = rng.choice([1, 1, _log_int(rng, 1, c["W"]), c["W"]])
        if kind == "read":
            c["ragged"] = rng.random() < 0.5
        most = {"tier1": 6e8, "append": 1e8, "read": 4e8}[kind]
    while c["B"] > 1 and work(c)["bytes"] > most:
        c["B"] = (c["B"] + 1) // 2
    while "N" in c and c["N"] > c["k"] and c["B"] * c["Hkv"] * c["N"] * c["Dh"] * _BYTES[c["kv"]] > 1.1e9:
        c["N"] = max(c["k"], c["N"] // 2)
    return c


# ------------------------------------------------------------- plain forms

def _blocks(x, block):
    """[B][H][R][D] as [B][H][ceil(R / block)][block][D], zero rows after the last."""
    B, H, R, D = x.shape
    n = -(-R // block)
    return torch.nn.functional.pad(x, (0, 0, 0, n * block - R)).view(B, H, n, block, D)


def _rows(per_block, block, R):
    """A block's value for each of its rows: [B][H][n] -> [B][H][R][1]."""
    return per_block.repeat_interleave(block, dim=2)[:, :, :R, None]


def _quantise(x, live, code, block):
    """x [B][H][R][D] fp32, live [B][1][R] -> codes [B][H][R][D], scales
    [B][H][ceil(R / block)] (1 where a block has no live row)."""
    most = _MOST[code]
    mag = torch.where(live[..., None] & x.isfinite(), x.abs(), torch.zeros((), device=x.device))
    a = _blocks(mag, block).amax(dim=(3, 4))
    m, e = torch.frexp(a)  # a = m 2^e, m in [1/2, 1)
    top, shift = math.frexp(most)
    e = torch.where(a > 0, e - shift + (m > top), -126).clamp(min=-126)
    scale = ((e + 127) << 23).to(torch.int32).view(F32)
    y = (x / _rows(scale, block, x.shape[2])).clamp(-most, most)
    if code == I8:
        y = torch.where(y.isnan(), torch.zeros((), device=x.device), y.round())
    some = _blocks(live[..., None], block).any(dim=(3, 4))
    return y.to(code), torch.where(some, scale, torch.ones((), device=x.device))


def _values(codes, scales, live, block):
    """fp32 values of the live rows, 0 elsewhere."""
    v = codes.to(F32) * _rows(scales, block, codes.shape[2])
    return torch.where(live[..., None], v, torch.zeros((), device=v.device))


def _count_mask(count, R):
    """[B][1][R]: the rows below each sequence's count."""
    return (torch.arange(R, device=count.device)[None, :] < count[:, None])[:, None]


def _plain_append(s):
    """The ring after this call's rows, in the state's own buffers."""
    W, T, block, count = s["win_k"].shape[2], s["new_k"].shape[2], s["block"], s["win_count"]
    slot = torch.arange(W, device=DEV)[None, :]
    age = (slot - count[:, None]) % W  # the appended row that slot takes, where it is below T
    fresh = (age < T)[:, None]
    old, live = _count_mask(count, W), _count_mask(count + T, W)
    touched = _blocks(fresh[..., None], block).any(dim=(3, 4))
    at = age.clamp(max=T - 1)[:, None, :, None]
    for x in ("k", "v"):
        codes, scales, new = s["win_" + x], s["win_" + x + "s"], s["new_" + x].to(F32)
        value = torch.where(fresh[..., None], new.gather(2, at.expand(-1, new.shape[1], -1, new.shape[3])),
                            _values(codes, scales, old, block))
        c, sc = _quantise(value, live, codes.dtype, block)
        put = _rows(touched.expand(-1, codes.shape[1], -1), block, W) & live[..., None]
        # the codes' bytes: a masked copy of 8-bit floats
        codes.view(torch.uint8).copy_(torch.where(put, c.view(torch.uint8), codes.view(torch.uint8)))
        scales.copy_(torch.where(touched, sc, scales))
    count += T


def _plain_attend(s):
    B, Hq, Dh = s["q"].shape
    Hkv, block = s["win_k"].shape[1], s["block"]
    k_len = s["k_len"] if s["k_len"] is not None else torch.full((B,), s["k"], device=DEV)
    live = torch.cat([_count_mask(k_len, s["k"]), _count_mask(s["win_count"], s["win_k"].shape[2])], dim=2)
    K, V = (torch.cat([_values(s["cme_" + x], s["cme_" + x + "s"], _count_mask(k_len, s["k"]), block),
                       _values(s["win_" + x], s["win_" + x + "s"], _count_mask(s["win_count"], s["win_k"].shape[2]), block)],
                      dim=2) for x in ("k", "v"))
    q = s["q"].view(B, Hkv, Hq // Hkv, Dh) * s["scale"]
    z = (q @ K.transpose(2, 3)).masked_fill(~live[:, :, None], -math.inf)
    top = z.amax(dim=3, keepdim=True)
    p = torch.exp(z - torch.where(top.isinf(), torch.zeros_like(top), top))
    den = p.sum(dim=3, keepdim=True)
    return ((p @ V) / torch.where(den > 0, den, torch.ones_like(den))).view(B, Hq, Dh)


# ------------------------------------------------------------------ inputs

class _Draws:
    """Seeded draws on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device=DEV, dtype=F32)

    def ints(self, lo, hi, B):
        return torch.randint(lo, hi + 1, (B,), generator=self.g, device=DEV, dtype=torch.int32)

    def rows(self, shape, kv, spread):
        """K or V rows of one type: N(0, 1), with channels of different sizes
        (keys more than values) as decoders have them."""
        B, H, R, D = shape
        x = self.normal(*shape)
        x *= torch.exp(spread * self.normal(1, H, 1, D))
        return x.to(_FLOAT[kv])


def _prepare_ring(c, d, count):
    """An 8-bit ring filled up to min(count, W)."""
    B, Hkv, Dh, W = c["B"], c["Hkv"], c["Dh"], c["W"]
    live = _count_mask(count, W)
    s = dict(block=c["block"], win_count=count)
    for x, spread in (("k", 0.7), ("v", 0.3)):
        rows = d.rows((B, Hkv, W, Dh), c["kv"], spread).to(F32)
        s["win_" + x], s["win_" + x + "s"] = _quantise(torch.where(live[..., None], rows, torch.zeros((), device=DEV)),
                                                       live, _CODE[c["code"]], c["block"])
    return s


def _prepare_decode(c, seed):
    d = _Draws(seed)
    B, Hq, Hkv, Dh, k, W = (c[x] for x in ("B", "Hq", "Hkv", "Dh", "k", "W"))
    if c["ragged"]:  # from a quarter of the rows up, rings from a quarter full to wrapped
        k_len, count = d.ints(max(1, k // 4), k, B), d.ints(max(1, W // 4), 2 * W, B)
    else:
        k_len, count = None, torch.full((B,), W + 3, dtype=torch.int32, device=DEV)
    s = _prepare_ring(c, d, count)
    all_rows = torch.full((B,), k, device=DEV)
    for x, spread in (("k", 0.7), ("v", 0.3)):
        s["cme_" + x], s["cme_" + x + "s"] = _quantise(d.rows((B, Hkv, k, Dh), c["kv"], spread).to(F32),
                                                       _count_mask(all_rows, k), _CODE[c["code"]], c["block"])
        if c["T"]:
            s["new_" + x] = d.rows((B, Hkv, c["T"], Dh), c["kv"], spread)
    s.update(k=k, k_len=k_len, q=d.normal(B, Hq, Dh), scale=1.0 / math.sqrt(Dh),
             out=torch.empty((B, Hq, Dh), dtype=F32, device=DEV))
    return s


_prepare_step = _prepare_attend = _prepare_decode


def _prepare_tier1(c, seed):
    d = _Draws(seed)
    B, Hkv, Dh, N, k = (c[x] for x in ("B", "Hkv", "Dh", "N", "k"))
    idx = torch.rand((B, N), generator=d.g, device=DEV).topk(k, dim=1).indices.sort(dim=1).values.to(torch.int32)
    n = -(-k // c["block"])
    s = dict(block=c["block"], k=k, idx=idx.contiguous(), k_len=d.ints(max(1, k // 4), k, B) if c["ragged"] else None)
    for x, spread in (("k", 0.7), ("v", 0.3)):
        s["cme_" + x] = d.rows((B, Hkv, N, Dh), c["kv"], spread)
        # rows past a sequence's count stay as they are
        s["out_" + x] = torch.zeros((B, Hkv, k, Dh), dtype=_CODE[c["code"]], device=DEV)
        s["out_" + x + "s"] = torch.zeros((B, Hkv, n), dtype=F32, device=DEV)
    return s


def _prepare_append(c, seed):
    d = _Draws(seed)
    B, Hkv, Dh, W, T = (c[x] for x in ("B", "Hkv", "Dh", "W", "T"))
    # a prefill starts an empty ring, a step finds one in use
    count = torch.zeros((B,), dtype=torch.int32, device=DEV) if T == W else d.ints(W // 2, 3 * W, B)
    s = _prepare_ring(c, d, count)
    for x, spread in (("k", 0.7), ("v", 0.3)):
        s["new_" + x] = d.rows((B, Hkv, T, Dh), c["kv"], spread)
    return s


def _prepare_read(c, seed):
    d = _Draws(seed)
    B, Hkv, Dh, W = (c[x] for x in ("B", "Hkv", "Dh", "W"))
    count = d.ints(max(1, W // 4), 2 * W, B) if c["ragged"] else torch.full((B,), W + 3, dtype=torch.int32, device=DEV)
    s = _prepare_ring(c, d, count)
    for x in ("k", "v"):
        s["out_" + x] = torch.zeros((B, Hkv, W, Dh), dtype=_FLOAT[c["kv"]], device=DEV)
    return s


def prepare(case, seed):
    return dict(kind=case["kind"], **globals()["_prepare_" + case["kind"]](case, seed))


# -------------------------------------------------------------------- runs

_RING = ("win_k", "win_v", "win_ks", "win_vs", "win_count")


def _workspace(s):
    """The decode workspace, made at the first pass and kept, as a serving
    program keeps it."""
    from paper_2609_25537_amd import cmc
    if "workspace" not in s:
        B, Hq, Dh = s["q"].shape
        s["workspace"] = cmc.decode_workspace_q8(B, Hq, s["win_k"].shape[1], Dh, s["k"], s["win_k"].shape[2], DEV)
    return s["workspace"]


def _run_step(s):
    if own:
        from paper_2609_25537_amd import cmc
        cmc.cmc_decode_step_q8(s["q"], s["cme_k"], s["cme_v"], s["cme_ks"], s["cme_vs"], s["k"], s["win_k"], s["win_v"],
                               s["win_ks"], s["win_vs"], s["win_count"], s["new_k"], s["new_v"], s["scale"], s["block"],
                               k_len=s["k_len"], out=s["out"], workspace=_workspace(s))
        out = s["out"]
    else:
        _plain_append(s)
        out = _plain_attend(s)
    return dict(out=out, **{x: s[x] for x in _RING})


def _run_attend(s):
    if own:
        from paper_2609_25537_amd import cmc
        return cmc.cmc_two_tier_decode_q8(s["q"], s["cme_k"], s["cme_v"], s["cme_ks"], s["cme_vs"], s["k"], s["win_k"],
                                          s["win_v"], s["win_ks"], s["win_vs"], s["win_count"], s["scale"], s["block"],
                                          k_len=s["k_len"], out=s["out"], workspace=_workspace(s))
    return _plain_attend(s)


def _run_tier1(s):
    out = {x: s[x] for x in ("out_k", "out_v", "out_ks", "out_vs")}
    if own:
        from paper_2609_25537_amd import cmc
        cmc.cmc_gather_tier1_q8(s["cme_k"], s["cme_v"], s["idx"], s["k"], s["block"], k_len=s["k_len"], **out)
        return out
    B, k = s["idx"].shape
    live = _count_mask(s["k_len"] if s["k_len"] is not None else torch.full((B,), k, device=DEV), k)
    some = _blocks(live[..., None], s["block"]).any(dim=(3, 4))
    for x in ("k", "v"):
        pool, codes, scales = s["cme_" + x], s["out_" + x], s["out_" + x + "s"]
        at = s["idx"].long()[:, None, :, None].expand(-1, pool.shape[1], -1, pool.shape[3])
        c, sc = _quantise(pool.gather(2, at).to(F32), live, codes.dtype, s["block"])
        codes.view(torch.uint8).copy_(torch.where(live[..., None], c.view(torch.uint8), codes.view(torch.uint8)))
        scales.copy_(torch.where(some, sc, scales))
    return out


def _run_append(s):
    if own:
        from paper_2609_25537_amd import cmc
        cmc.cmc_window_append_q8(s["win_k"], s["win_v"], s["win_ks"], s["win_vs"], s["win_count"], s["new_k"], s["new_v"],
                                 s["block"])
    else:
        _plain_append(s)
    return {x: s[x] for x in _RING}


def _run_read(s):
    out = {x: s[x] for x in ("out_k", "out_v")}
    if own:
        from paper_2609_25537_amd import cmc
        cmc.cmc_cache_read_q8(s["win_k"], s["win_v"], s["win_ks"], s["win_vs"], s["block"], count=s["win_count"], **out)
        return out
    W, count = s["win_k"].shape[2], s["win_count"]
    live = _count_mask(count, W)
    first = torch.where(count > W, count % W, torch.zeros_like(count))
    row = ((first[:, None] + torch.arange(W, device=DEV)[None, :]) % W)[:, None, :, None]
    for x in ("k", "v"):
        v = _values(s["win_" + x], s["win_" + x + "s"], live, s["block"])
        v = v.gather(2, row.expand(-1, v.shape[1], -1, v.shape[3])).to(out["out_" + x].dtype)
        out["out_" + x].copy_(torch.where(live[..., None], v, out["out_" + x]))
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
    ragged = c.get("ragged", False)
    full = 0.8571 if ragged else 1.0  # mean of min(count, W) / W for counts from W / 4 to 2 W
    if c["kind"] in ("step", "attend"):
        keys = c["k"] * (0.625 if ragged else 1.0) + c["W"] * full
        wrote = c["T"] * (_BYTES[c["kv"]] + 1) if c["T"] else 0
        return {"bytes": B * (row * (keys * (1 + 4.0 / (c["block"] * Dh)) + wrote) + 8 * c["Hq"] * Dh),
                "flops": 4.0 * B * c["Hq"] * keys * Dh}
    if c["kind"] == "tier1":
        keys = c["k"] * (0.625 if ragged else 1.0)
        return {"bytes": B * (row * keys * (_BYTES[c["kv"]] + 1 + 4.0 / (c["block"] * Dh)) + 4 * keys),
                "flops": 3.0 * B * row * keys}
    if c["kind"] == "append":
        # a block's other rows are read for its scale
        old = min(c["W"], (c["T"] - 1) // c["block"] * c["block"] + c["block"]) - c["T"] if c["T"] < c["W"] else 0
        return {"bytes": B * row * (c["T"] * (_BYTES[c["kv"]] + 1) + max(old, 0) + 4.0 / Dh),
                "flops": 3.0 * B * row * (c["T"] + max(old, 0))}
    return {"bytes": B * row * c["W"] * full * (1 + _BYTES[c["kv"]] + 4.0 / (c["block"] * Dh)),
            "flops": 1.0 * B * row * c["W"] * full}


# ------------------------------------------------------------------- exact

def _exact_codes(x, code):
    """One block's rows (fp64, [H][rows][D]) to (codes, scale [H]), from the
    definition: the least power of two, then the nearest code."""
    most = 448.0 if code == E4M3 else 127.0
    a = torch.where(x.isfinite(), x.abs(), torch.zeros_like(x)).flatten(1).amax(dim=1)
    e = torch.full_like(a, -126.0)
    some = a > 0
    e[some] = torch.ceil(torch.log2(a[some] / most)) - 1  # log2 may be off by a rounding: count up from below
    e = e.clamp(min=-126.0)
    for _ in range(3):
        e = e + (a > most * torch.exp2(e)).double()
    s = torch.exp2(e)
    y = (x / s[:, None, None]).clamp(-most, most)
    if code == I8:
        return torch.round(y), s
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, s


def _exact_append(s):
    """The ring after the append, block by block: fp64 codes and scales."""
    W, T, block = s["win_k"].shape[2], s["new_k"].shape[2], s["block"]
    r = {x: s[x].double() for x in _RING[:4]}
    r["win_count"] = s["win_count"].long() + T
    for b, count in enumerate(s["win_count"].tolist()):
        slots = [(count + t) % W for t in range(T)]
        filled = min(count + T, W)
        for j in sorted({x // block for x in slots}):
            lo, hi = j * block, min((j + 1) * block, filled)
            mine = [(t, x - lo) for t, x in enumerate(slots) if lo <= x < hi]
            for x in ("k", "v"):
                rows = r["win_" + x][b, :, lo:hi] * r["win_" + x + "s"][b, :, j, None, None]
                rows[:, [p for _, p in mine]] = s["new_" + x][b][:, [t for t, _ in mine]].double()
                r["win_" + x][b, :, lo:hi], r["win_" + x + "s"][b, :, j] = _exact_codes(rows, s["win_k"].dtype)
    return r


def _exact_attend(s, ring):
    """Each sequence's attention over its own list of keys, in fp64."""
    B, Hq, Dh = s["q"].shape
    Hkv, W, block = s["win_k"].shape[1], s["win_k"].shape[2], s["block"]
    out = torch.zeros((B, Hkv, Hq // Hkv, Dh), dtype=torch.float64, device=DEV)
    for b in range(B):
        n = s["k"] if s["k_len"] is None else int(s["k_len"][b])
        w = min(int(ring["win_count"][b]), W)
        lists = []
        for x in ("k", "v"):
            parts = []
            for codes, scales, rows in ((s["cme_" + x][b], s["cme_" + x + "s"][b], n), (ring["win_" + x][b], ring["win_" + x + "s"][b], w)):
                at = torch.arange(rows, device=DEV) // block
                parts.append(codes[:, :rows].double() * scales.double()[:, at, None])
            lists.append(torch.cat(parts, dim=1))
        q = s["q"][b].double().view(Hkv, Hq // Hkv, Dh)
        out[b] = torch.softmax(torch.matmul(q, lists[0].transpose(1, 2).contiguous()) / math.sqrt(Dh), dim=2) @ lists[1]
    return out.view(B, Hq, Dh)


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind in ("step", "append"):
        if kind == "append" and case["B"] * case["T"] > 40000:
            return None
        ring = _exact_append(s)
        return dict(out=_exact_attend(s, ring), **ring) if kind == "step" else ring
    if kind == "attend":
        return _exact_attend(s, {x: s[x] for x in _RING})
    if kind == "tier1":
        r = {x: s[x].double() for x in ("out_k", "out_v", "out_ks", "out_vs")}
        for b in range(case["B"]):
            n = s["k"] if s["k_len"] is None else int(s["k_len"][b])
            at = s["idx"][b, :n].long()
            for j in range(-(-n // s["block"])):
                lo, hi = j * s["block"], min((j + 1) * s["block"], n)
                for x in ("k", "v"):
                    rows = s["cme_" + x][b][:, at[lo:hi]].double()
                    r["out_" + x][b, :, lo:hi], r["out_" + x + "s"][b, :, j] = _exact_codes(rows, s["out_k"].dtype)
        return r
    r = {x: s[x].double() for x in ("out_k", "out_v")}
    W = s["win_k"].shape[2]
    for b, count in enumerate(s["win_count"].tolist()):
        n, first = min(count, W), count % W if count > W else 0
        at = (first + torch.arange(n, device=DEV)) % W
        for x in ("k", "v"):
            r["out_" + x][b, :, :n] = s["win_" + x][b][:, at].double() * s["win_" + x + "s"][b].double()[:, at // s["block"], None]
    return r
