"""The 8-bit cache's calls on the CPU: what they refuse, before anything is
launched; the wrappers' own checks; and the fp64 reference's rounding against
torch's casts."""
import itertools

import numpy as np
import pytest
import torch

from paper_2609_25537_amd import cmc
from tests import q8_ref

INV, UNS, WS, OK = cmc.CMC_ERR_INVALID_ARGUMENT, cmc.CMC_ERR_UNSUPPORTED, cmc.CMC_ERR_WORKSPACE_TOO_SMALL, cmc.CMC_OK
FAKE = 1 << 20  # 16-byte aligned non-null address, never dereferenced: the calls fail validation first


def _gather(**kw):
    a = dict(ck=FAKE, cv=FAKE, kd=cmc.CMC_BF16, idx=FAKE, kl=FAKE, stride=8, B=2, Hkv=2, N=16, k=8, Dh=128, code=cmc.CMC_E4M3,
             block=32, ok=FAKE, ov=FAKE, oks=FAKE, ovs=FAKE, s=None)
    a.update(kw)
    return cmc.lib().cmc_gather_tier1_q8(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(kd=cmc.CMC_I8), UNS), (dict(kd=9), UNS), (dict(code=cmc.CMC_BF16), UNS), (dict(code=-1), UNS),
    (dict(block=16), UNS), (dict(block=0), UNS), (dict(block=256), UNS), (dict(Dh=96), UNS), (dict(Hkv=0), INV),
    (dict(B=-1), INV), (dict(k=-1), INV), (dict(N=-1), INV), (dict(stride=7), INV), (dict(idx=None, k=17), INV),
    (dict(N=0), INV), (dict(B=65536), UNS), (dict(Hkv=65536), UNS), (dict(k=(1 << 26) + 1, idx=None, N=1 << 30), UNS),
    (dict(ck=None), INV), (dict(oks=None), INV), (dict(ovs=FAKE + 4), UNS), (dict(ok=FAKE + 8), UNS), (dict(idx=FAKE + 4), UNS),
])
def test_gather_refusals(kw, code):
    assert _gather(**kw) == code
    assert cmc.last_error()


def test_gather_nothing_to_do():
    assert _gather(B=0) == OK and _gather(k=0) == OK
    assert _gather(k=0, N=0, ck=None, ok=None) == OK


def _app(**kw):
    a = dict(wk=FAKE, wv=FAKE, wks=FAKE, wvs=FAKE, code=cmc.CMC_I8, block=32, wc=FAKE, nk=FAKE, nv=FAKE, nd=cmc.CMC_F32, B=2,
             Hkv=2, W=8, Dh=128, T=1, s=None)
    a.update(kw)
    return cmc.lib().cmc_window_append_q8(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(T=0), INV), (dict(T=9), INV), (dict(Dh=80), UNS), (dict(Hkv=0), INV), (dict(nk=None), INV), (dict(wks=None), INV),
    (dict(wc=FAKE + 4), UNS), (dict(nd=cmc.CMC_E4M3), UNS), (dict(code=cmc.CMC_F32), UNS), (dict(block=33), UNS),
    (dict(W=-1), INV), (dict(B=70000), UNS), (dict(W=(1 << 26) + 1), UNS), (dict(wvs=FAKE + 8), UNS),
])
def test_append_refusals(kw, code):
    assert _app(**kw) == code
    assert cmc.last_error()


def test_append_nothing_to_do():
    assert _app(W=0, T=0) == OK and _app(B=0) == OK


def _read(**kw):
    a = dict(k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, code=cmc.CMC_E4M3, block=64, n=FAKE, B=1, Hkv=2, R=8, Dh=64, od=cmc.CMC_BF16,
             ok=FAKE, ov=FAKE, s=None)
    a.update(kw)
    return cmc.lib().cmc_cache_read_q8(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(od=cmc.CMC_E4M3), UNS), (dict(code=cmc.CMC_F32), UNS), (dict(block=48), UNS), (dict(Dh=32), UNS), (dict(R=-1), INV),
    (dict(ks=None), INV), (dict(ov=None), INV), (dict(ok=FAKE + 4), UNS), (dict(n=FAKE + 4), UNS), (dict(Hkv=0), INV),
])
def test_read_refusals(kw, code):
    assert _read(**kw) == code
    assert cmc.last_error()


def test_read_nothing_to_do():
    assert _read(B=0) == OK and _read(R=0, k=None) == OK


def _step(**kw):
    a = dict(q=FAKE, ck=FAKE, cv=FAKE, cks=FAKE, cvs=FAKE, kl=FAKE, k=4, wk=FAKE, wv=FAKE, wks=FAKE, wvs=FAKE, wc=FAKE, W=8,
             nk=FAKE, nv=FAKE, T=1, nd=cmc.CMC_BF16, code=cmc.CMC_E4M3, block=32, B=1, Hq=8, Hkv=2, Dh=128, N=16, scale=0.1,
             out=FAKE, ws=FAKE, wsb=1 << 30, s=None)
    a.update(kw)
    return cmc.lib().cmc_decode_step_q8(*a.values())


def _dec(**kw):
    a = dict(q=FAKE, ck=FAKE, cv=FAKE, cks=FAKE, cvs=FAKE, kl=None, k=4, wk=FAKE, wv=FAKE, wks=FAKE, wvs=FAKE, wc=FAKE, W=8,
             code=cmc.CMC_E4M3, block=32, B=1, Hq=8, Hkv=2, Dh=128, N=16, scale=0.1, out=FAKE, ws=FAKE, wsb=1 << 30, s=None)
    a.update(kw)
    return cmc.lib().cmc_two_tier_decode_q8(*a.values())


@pytest.mark.parametrize("call", [_step, _dec])
@pytest.mark.parametrize("kw,code", [
    (dict(Hq=6, Hkv=4), INV), (dict(Hq=12, Hkv=4), UNS), (dict(Hq=0), INV), (dict(Dh=96), UNS), (dict(k=17), INV),
    (dict(k=-1), INV), (dict(code=cmc.CMC_BF16), UNS), (dict(block=8), UNS), (dict(wsb=64), WS), (dict(ws=None), WS),
    (dict(out=FAKE + 8), UNS), (dict(wc=None), INV), (dict(wks=None), INV), (dict(cvs=None), INV), (dict(q=None), INV),
    (dict(scale=float("nan")), INV), (dict(scale=float("inf")), INV), (dict(B=-1), INV), (dict(B=65536), UNS),
    (dict(N=(1 << 26) + 1), UNS), (dict(W=(1 << 26) + 1), UNS), (dict(cks=FAKE + 4), UNS), (dict(ws=FAKE + 8), UNS),
])
def test_decode_refusals(call, kw, code):
    assert call(**kw) == code
    assert cmc.last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(T=0), INV), (dict(T=9), INV), (dict(T=-1), INV), (dict(nk=None), INV), (dict(nd=cmc.CMC_I8), UNS),
    (dict(nv=FAKE + 8), UNS), (dict(W=0, k=0), INV),
])
def test_step_refusals(kw, code):
    assert _step(**kw) == code
    assert cmc.last_error()


def test_decode_empty_batch_and_workspace_query():
    assert _dec(B=0) == OK and _step(B=0) == OK
    f = cmc.cmc_decode_q8_workspace_bytes
    assert f(1, 32, 8, 128, 256, 512) > 0
    for bad in ((1, 32, 7, 128, 256, 512), (1, 32, 8, 100, 256, 512), (-1, 32, 8, 128, 1, 1), (1, 32, 8, 128, -1, 5)):
        assert f(*bad) == 0
    # partials are kept for as many splits as the merge can hold
    assert f(1, 32, 8, 128, 0, 1 << 26) < 1 << 24


# ---------------------------------------------------------------- wrappers

E4 = torch.float8_e4m3fn


def _cache(B=1, H=2, R=40, Dh=64, block=32, code=E4):
    n = -(-R // block)
    return [torch.zeros((B, H, R, Dh)).to(code), torch.zeros((B, H, R, Dh)).to(code), torch.zeros((B, H, n)),
            torch.zeros((B, H, n))]


def test_wrappers_refuse_what_does_not_fit():
    pool = torch.zeros((1, 2, 50, 64), dtype=torch.bfloat16)
    new = torch.zeros((1, 2, 1, 64), dtype=torch.bfloat16)
    count = torch.zeros((1,), dtype=torch.int32)
    q = torch.zeros((1, 4, 64))
    w = _cache()
    g, a, r, d, s = (cmc.cmc_gather_tier1_q8, cmc.cmc_window_append_q8, cmc.cmc_cache_read_q8, cmc.cmc_two_tier_decode_q8,
                     cmc.cmc_decode_step_q8)
    bad = [
        lambda: g(pool[:, :, ::2], pool[:, :, ::2], None, 8, 32), lambda: g(pool, pool.float(), None, 8, 32),
        lambda: g(pool, pool, None, 8, 0), lambda: g(pool, pool, count.view(1, 1).long(), 1, 32),
        lambda: g(pool, pool, None, 8, 32, out_k=w[0]), lambda: g(pool, pool, None, 40, 32, out_k=w[0], out_ks=w[2][:, :, :1]),
        lambda: g(pool, pool, None, 8, 32, k_len=count.long()),
        lambda: a(*w, count.long(), new, new, 32), lambda: a(*w, count, new, new, 64), lambda: a(*w, count, new, new.float(), 32),
        lambda: a(w[0], w[1].to(torch.int8), w[2], w[3], count, new, new, 32),
        lambda: a(*w, count, new.expand(1, 2, 3, 64), new.expand(1, 2, 3, 64), 32),
        lambda: a(w[0].transpose(1, 2), w[1].transpose(1, 2), w[2], w[3], count, new, new, 32),
        lambda: r(*w, 32, out_k=torch.zeros((1, 2, 39, 64))), lambda: r(*w, 32, count=count.long()), lambda: r(*w, -1),
        lambda: d(q.double(), *w, 40, *w, count, 0.1, 32), lambda: d(q, *w, 40, *_cache(code=torch.int8), count, 0.1, 32),
        lambda: d(q, *w, 40, *_cache(H=1), count, 0.1, 32), lambda: d(q, *w, 40, *w, count, 0.1, 64),
        lambda: d(q, *w, 40, *w, count, 0.1, 32, k_len=count.long()), lambda: d(q, *w, 40, *w, count, 0.1, 32, out=q[0]),
        lambda: s(q, *w, 40, *w, count, new, new.float(), 0.1, 32), lambda: s(q, *w, 40, *w, count, new[0], new[0], 0.1, 32),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was taken")
    with pytest.raises(TypeError):  # codes of no 8-bit type
        x = [t.float() for t in w]
        cmc._code_dtype(x[0])


def test_wrappers_refuse_a_workspace_with_gaps():
    """Every second byte of a buffer that ends where the workspace would go on."""
    w, q, count = _cache(), torch.zeros((1, 4, 64)), torch.zeros((1,), dtype=torch.int32)
    new = torch.zeros((1, 2, 1, 64), dtype=torch.bfloat16)
    ws = torch.zeros(2 * cmc.cmc_decode_q8_workspace_bytes(1, 4, 2, 64, 40, 40), dtype=torch.uint8)[::2]
    with pytest.raises(ValueError, match="workspace must be contiguous"):
        cmc.cmc_two_tier_decode_q8(q, *w, 40, *w, count, 0.1, 32, workspace=ws)
    with pytest.raises(ValueError, match="workspace must be contiguous"):
        cmc.cmc_decode_step_q8(q, *w, 40, *w, count, new, new, 0.1, 32, workspace=ws)


def test_wrappers_refuse_host_tensors():
    w = _cache()
    with pytest.raises(Exception, match="device|CUDA|HIP|NVIDIA|GPU"):
        cmc.cmc_cache_read_q8(*w, 32)


# --------------------------------------------------------------- reference

def test_reference_rounding_is_the_types():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(20000) * s for s in (0.001, 0.02, 1.0, 50.0)]).astype(np.float32)
    x = np.clip(x, -448, 448)
    assert (q8_ref.round_code(x, "e4m3") == torch.from_numpy(x).to(E4).to(torch.float64).numpy()).all()
    y = np.clip(x, -127, 127)
    assert (q8_ref.round_code(y, "i8") == torch.from_numpy(y).round().to(torch.float64).numpy()).all()


def test_reference_scale_is_the_least():
    for code, a in itertools.product(("e4m3", "i8"), (0.0, 1e-45, 1e-30, 0.3, 1.0, 127.0, 127.5, 448.0, 449.0, 3e38)):
        s = q8_ref.scale_of(np.array([a, -a / 2, np.inf, np.nan]), code)
        assert a <= q8_ref.MOST[code] * s and (s == 2.0 ** -126 or a > q8_ref.MOST[code] * s / 2)
        assert np.frexp(s)[0] == 0.5


def test_reference_attention_is_softmax():
    rng = np.random.default_rng(1)
    q, K, V = rng.standard_normal(16), rng.standard_normal((9, 16)), rng.standard_normal((9, 16))
    t = [torch.from_numpy(v)[None] for v in (q[None], K, V)]
    want = torch.nn.functional.scaled_dot_product_attention(*t, scale=0.3)[0, 0].numpy()
    assert np.abs(q8_ref.attend(q, K, V, 0.3)[0] - want).max() < 1e-13
