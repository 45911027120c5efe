"""Calls given a stream that is not the current one, which meanwhile has long work
of its own queued, with the outputs and workspaces left to the call: results as
on the current stream, also where that stream's freed memory holds other data."""
import torch
import pytest

from paper_2609_25537_amd import cmc
from tests.gpu_util import DEV, say

pytestmark = pytest.mark.gpu


def _inputs(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)
    B, Hq, Hkv, Dh, N, k, W = 2, 16, 4, 128, 900, 500, 700
    r = dict(k=k, q=n(B, Hq, Dh), pk=n(B, Hkv, N, Dh), pv=n(B, Hkv, N, Dh), keys=n(B, N, 64), qv=n(B, 64),
             win=[n(B, Hkv, W, Dh), n(B, Hkv, W, Dh)], new=[n(B, Hkv, 1, Dh), n(B, Hkv, 1, Dh)],
             count=torch.full((B,), W + 5, dtype=torch.int32, device=DEV))
    zero = torch.zeros((B,), dtype=torch.int32, device=DEV)
    r["ring8"] = [torch.zeros((B, Hkv, W, Dh), dtype=torch.int8, device=DEV) for _ in range(2)]
    r["ring8"] += [torch.zeros((B, Hkv, -(-W // 32)), device=DEV) for _ in range(2)]
    cmc.cmc_window_append_q8(*r["ring8"], zero, *r["win"], 32)
    r["count8"] = zero + 5
    return r


def _run(r, stream):
    """Selection, both gathers, both steps, both attentions and the read back."""
    idx = cmc.cmc_select_cmes(r["keys"], r["qv"], r["k"], stream=stream)
    gk, gv = cmc.cmc_gather_tier1(r["pk"], r["pv"], idx, r["k"], stream=stream)
    tier8 = cmc.cmc_gather_tier1_q8(r["pk"], r["pv"], idx, r["k"], 32, dtype=torch.int8, stream=stream)
    out = [idx, gk, gv, *tier8]
    for _ in range(3):
        out.append(cmc.cmc_decode_step(r["q"], r["pk"], r["pv"], idx, r["k"], *r["win"], r["count"], *r["new"], 0.09,
                                       stream=stream))
        out.append(cmc.cmc_decode_step_q8(r["q"], *tier8, r["k"], *r["ring8"], r["count8"], *r["new"], 0.09, 32, stream=stream))
        out.append(cmc.cmc_two_tier_decode(r["q"], r["pk"], r["pv"], idx, r["k"], *r["win"], r["count"], 0.09, stream=stream))
        out.append(cmc.cmc_two_tier_decode_q8(r["q"], *tier8, r["k"], *r["ring8"], r["count8"], 0.09, 32, stream=stream))
    out += cmc.cmc_cache_read_q8(*r["ring8"], 32, count=r["count8"], stream=stream)
    return out + [r["count"], r["count8"], *r["win"], *r["ring8"]]


@pytest.mark.parametrize("raw", [False, True])
def test_calls_on_a_side_stream(raw):
    want = [t.clone() for t in _run(_inputs(3), None)]
    r = _inputs(3)
    side = torch.cuda.Stream()
    a = torch.randn(4096, 4096, device=DEV).to(torch.bfloat16)
    b = torch.empty_like(a)
    torch.mm(a, a, out=b)
    torch.cuda.synchronize()
    say("side stream, raw handle" if raw else "side stream")
    for _ in range(100):  # tens of milliseconds on the current stream
        torch.mm(a, a, out=b)
    for n in (1 << 12, 1 << 16, 1 << 20, 1 << 22):  # its freed memory, of the outputs' and workspaces' sizes
        junk = [torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(8)]
        del junk
    got = _run(r, side.cuda_stream if raw else side)
    side.synchronize()
    for _ in range(8):  # new work of the current stream, in whatever the calls have dropped
        torch.full((1 << 20,), 0xFF, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    for i, (x, y) in enumerate(zip(got, want)):
        assert torch.equal(x, y), i
