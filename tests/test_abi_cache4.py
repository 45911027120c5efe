"""The 4-bit cache's calls and cmc_norm_rope on the CPU: what they refuse, before
anything is launched; the wrappers' own checks; on which stream a wrapper makes its
outputs; and the fp64 reference's rounding."""
import numpy as np
import pytest
import torch

from paper_2609_25537_amd import cmc
from tests import q4_ref
from tests.test_abi_streams import MAIN, Stream, made  # noqa: F401  (a fixture)

INV, UNS, WS, OK = cmc.CMC_ERR_INVALID_ARGUMENT, cmc.CMC_ERR_UNSUPPORTED, cmc.CMC_ERR_WORKSPACE_TOO_SMALL, cmc.CMC_OK
FAKE = 1 << 20  # 16-byte aligned non-null address, never dereferenced: the calls fail validation first
MANY = (1 << 24) + 1


def _gather(**kw):
    a = dict(ck=FAKE, cv=FAKE, kd=cmc.CMC_BF16, idx=FAKE, kl=FAKE, stride=8, B=2, Hkv=2, N=16, k=8, Dh=128,
             ok=FAKE, ov=FAKE, oks=FAKE, ovs=FAKE, s=None)
    a.update(kw)
    return cmc.lib().cmc_gather_tier1_q4(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(kd=cmc.CMC_I8), UNS), (dict(kd=9), UNS), (dict(Dh=96), UNS), (dict(Dh=32), UNS), (dict(Hkv=0), INV), (dict(B=-1), INV),
    (dict(k=-1), INV), (dict(N=-1), INV), (dict(stride=7), INV), (dict(idx=None, k=17), INV), (dict(N=0), INV),
    (dict(B=65536), UNS), (dict(Hkv=65536), UNS), (dict(k=MANY, idx=None, N=1 << 30), UNS), (dict(ck=None), INV),
    (dict(oks=None), INV), (dict(ovs=FAKE + 4), UNS), (dict(ok=FAKE + 8), UNS), (dict(idx=FAKE + 4), UNS), (dict(kl=FAKE + 4), UNS),
])
def test_gather_refusals(kw, code):
    assert _gather(**kw) == code
    assert cmc.last_error()


def _app(**kw):
    a = dict(wk=FAKE, wv=FAKE, wks=FAKE, wvs=FAKE, wc=FAKE, nk=FAKE, nv=FAKE, nd=cmc.CMC_F32, B=2, Hkv=2, W=8, Dh=128, T=1, s=None)
    a.update(kw)
    return cmc.lib().cmc_window_append_q4(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(T=0), INV), (dict(T=9), INV), (dict(Dh=80), UNS), (dict(Hkv=0), INV), (dict(nk=None), INV), (dict(wks=None), INV),
    (dict(wc=FAKE + 4), UNS), (dict(nd=cmc.CMC_E4M3), UNS), (dict(W=-1), INV), (dict(B=70000), UNS), (dict(W=MANY), UNS),
    (dict(wvs=FAKE + 8), UNS), (dict(wc=None), INV),
])
def test_append_refusals(kw, code):
    assert _app(**kw) == code
    assert cmc.last_error()


def _read(**kw):
    a = dict(k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, n=FAKE, B=1, Hkv=2, R=8, rows=8, Dh=64, od=cmc.CMC_BF16, ok=FAKE, ov=FAKE, s=None)
    a.update(kw)
    return cmc.lib().cmc_cache_read_q4(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(od=cmc.CMC_E4M3), UNS), (dict(Dh=32), UNS), (dict(R=-1), INV), (dict(rows=9), INV), (dict(rows=-1), INV),
    (dict(ks=None), INV), (dict(ov=None), INV), (dict(ok=FAKE + 4), UNS), (dict(n=FAKE + 4), UNS), (dict(Hkv=0), INV),
    (dict(R=MANY), UNS),
])
def test_read_refusals(kw, code):
    assert _read(**kw) == code
    assert cmc.last_error()


def _step(**kw):
    a = dict(q=FAKE, ck=FAKE, cv=FAKE, cks=FAKE, cvs=FAKE, kl=FAKE, k=4, wk=FAKE, wv=FAKE, wks=FAKE, wvs=FAKE, wc=FAKE, W=8,
             nk=FAKE, nv=FAKE, T=1, nd=cmc.CMC_BF16, B=1, Hq=8, Hkv=2, Dh=128, N=16, scale=0.1, out=FAKE, ws=FAKE,
             wsb=1 << 30, s=None)
    a.update(kw)
    return cmc.lib().cmc_decode_step_q4(*a.values())


def _dec(**kw):
    a = dict(q=FAKE, ck=FAKE, cv=FAKE, cks=FAKE, cvs=FAKE, kl=None, k=4, wk=FAKE, wv=FAKE, wks=FAKE, wvs=FAKE, wc=FAKE, W=8,
             B=1, Hq=8, Hkv=2, Dh=128, N=16, scale=0.1, out=FAKE, ws=FAKE, wsb=1 << 30, s=None)
    a.update(kw)
    return cmc.lib().cmc_two_tier_decode_q4(*a.values())


@pytest.mark.parametrize("call", [_step, _dec])
@pytest.mark.parametrize("kw,code", [
    (dict(Hq=6, Hkv=4), INV), (dict(Hq=12, Hkv=4), UNS), (dict(Hq=0), INV), (dict(Dh=96), UNS), (dict(k=17), INV),
    (dict(k=-1), INV), (dict(wsb=64), WS), (dict(ws=None), WS), (dict(out=FAKE + 8), UNS), (dict(wc=None), INV),
    (dict(wks=None), INV), (dict(cvs=None), INV), (dict(q=None), INV), (dict(scale=float("nan")), INV),
    (dict(scale=float("inf")), INV), (dict(B=-1), INV), (dict(B=65536), UNS), (dict(N=MANY), UNS), (dict(W=MANY), UNS),
    (dict(cks=FAKE + 4), UNS), (dict(ws=FAKE + 8), UNS), (dict(W=0, k=0), INV),
])
def test_decode_refusals(call, kw, code):
    assert call(**kw) == code
    assert cmc.last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(T=0), INV), (dict(T=9), INV), (dict(T=-1), INV), (dict(nk=None), INV), (dict(nd=cmc.CMC_I8), UNS), (dict(nv=FAKE + 8), UNS),
])
def test_step_refusals(kw, code):
    assert _step(**kw) == code
    assert cmc.last_error()


def _rope(**kw):
    a = dict(q=FAKE, qs=1024, k=FAKE, ks=512, v=FAKE, vs=512, d=cmc.CMC_BF16, pos=FAKE, f=FAKE, rot=128, i=0, qw=FAKE, kw_=FAKE,
             eps=1e-6, B=2, T=3, Hq=8, Hkv=4, Dh=128, oq=FAKE, qd=cmc.CMC_F32, ok=FAKE, ov=FAKE, kd=cmc.CMC_BF16, s=None)
    a.update(kw)
    return cmc.lib().cmc_norm_rope(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(d=cmc.CMC_I8), UNS), (dict(qd=7), UNS), (dict(kd=cmc.CMC_E4M3), UNS), (dict(Dh=96), UNS), (dict(rot=24), UNS),
    (dict(rot=130), INV), (dict(rot=-16), INV), (dict(B=-1), INV), (dict(T=-1), INV), (dict(Hq=-1), INV), (dict(Hkv=-1), INV),
    (dict(Hq=65536), UNS), (dict(Hkv=65536), UNS), (dict(B=1 << 16, T=1 << 15), UNS), (dict(eps=-1.0), INV),
    (dict(eps=float("inf")), INV), (dict(eps=float("nan")), INV), (dict(qs=1023), INV), (dict(ks=516), INV), (dict(vs=256), INV),
    (dict(q=None), INV), (dict(oq=None), INV), (dict(k=None), INV), (dict(ok=None), INV), (dict(ov=None), INV),
    (dict(pos=None), INV), (dict(f=None), INV), (dict(q=FAKE + 8), UNS), (dict(pos=FAKE + 2), UNS), (dict(f=FAKE + 4), UNS),
    (dict(kw_=FAKE + 8), UNS), (dict(ov=FAKE + 2), UNS),
])
def test_rope_refusals(kw, code):
    assert _rope(**kw) == code
    assert cmc.last_error()


def test_nothing_to_do():
    assert _gather(B=0) == OK and _gather(k=0) == OK and _gather(k=0, N=0, ck=None, ok=None) == OK
    assert _app(W=0, T=0) == OK and _app(B=0) == OK
    assert _read(B=0) == OK and _read(R=0, rows=0, k=None) == OK and _read(rows=0) == OK
    assert _dec(B=0) == OK and _step(B=0) == OK
    assert _rope(B=0) == OK and _rope(T=0) == OK and _rope(Hq=0, k=None, v=None) == OK and _rope(Hq=0, Hkv=0) == OK


def test_workspace_query():
    q = cmc.cmc_decode_q4_workspace_bytes
    assert q(1, 32, 8, 128, 256, 512) > 0
    assert q(-1, 32, 8, 128, 1, 1) == q(1, 0, 8, 128, 1, 1) == q(1, 9, 8, 128, 1, 1) == q(1, 32, 8, 96, 1, 1) == q(1, 8, 8, 64, -1, 1) == 0


def _t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


def _c(R=8, Dh=64, B=1):
    u8 = torch.uint8
    return [_t(B, 2, R, Dh // 2, dtype=u8), _t(B, 2, R, Dh // 2, dtype=u8), _t(B, 2, R, Dh // 32, dtype=u8), _t(B, 2, R, Dh // 32, dtype=u8)]


def _with(c, i, t):
    return c[:i] + [t] + c[i + 1:]


N, Q, NEW = _t(1, dtype=torch.int32), _t(1, 4, 64), _t(1, 2, 1, 64)
X, POS, F = _t(2, 3, 4, 64), _t(2, 3, dtype=torch.int32), _t(32)

WRAPPER_REFUSALS = {
    "codes not uint8": lambda: cmc.cmc_window_append_q4(*_with(_c(), 0, _t(1, 2, 8, 32)), N, NEW, NEW),
    "scales' shape": lambda: cmc.cmc_window_append_q4(*_with(_c(), 2, _t(1, 2, 8, 3, dtype=torch.uint8)), N, NEW, NEW),
    "strided codes": lambda: cmc.cmc_window_append_q4(*[x.expand(2, -1, -1, -1)[:1].transpose(1, 2).contiguous().transpose(1, 2)
                                                        for x in _c()], N, NEW, NEW),
    "counts int64": lambda: cmc.cmc_window_append_q4(*_c(), N.long(), NEW, NEW),
    "new rows' heads": lambda: cmc.cmc_window_append_q4(*_c(), N, _t(1, 3, 1, 64), _t(1, 3, 1, 64)),
    "pool": lambda: cmc.cmc_gather_tier1_q4(_t(1, 2, 8, 64), _t(1, 2, 9, 64), None, 4),
    "k below 0": lambda: cmc.cmc_gather_tier1_q4(_t(1, 2, 8, 64), _t(1, 2, 8, 64), None, -1),
    "idx": lambda: cmc.cmc_gather_tier1_q4(_t(1, 2, 8, 64), _t(1, 2, 8, 64), _t(1, 4), 4),
    "gathered shape": lambda: cmc.cmc_gather_tier1_q4(_t(1, 2, 8, 64), _t(1, 2, 8, 64), None, 4, out_k=_c()[0]),
    "rows below 0": lambda: cmc.cmc_cache_read_q4(*_c(), rows=-1),
    "rows and out_k": lambda: cmc.cmc_cache_read_q4(*_c(), rows=3, out_k=_t(1, 2, 4, 64)),
    "read types": lambda: cmc.cmc_cache_read_q4(*_c(), out_k=_t(1, 2, 4, 64), out_v=_t(1, 2, 4, 64, dtype=torch.bfloat16)),
    "q": lambda: cmc.cmc_two_tier_decode_q4(Q.double(), *_c(), 8, *_c(), N, 0.1),
    "Dh": lambda: cmc.cmc_two_tier_decode_q4(Q, *_c(Dh=128), 8, *_c(), N, 0.1),
    "ring's Dh": lambda: cmc.cmc_two_tier_decode_q4(Q, *_c(), 8, *_c(Dh=128), N, 0.1),
    "no count": lambda: cmc.cmc_two_tier_decode_q4(Q, *_c(), 8, *_c(), None, 0.1),
    "k_len": lambda: cmc.cmc_two_tier_decode_q4(Q, *_c(), 8, *_c(), N, 0.1, k_len=_t(2, dtype=torch.int32)),
    "out": lambda: cmc.cmc_two_tier_decode_q4(Q, *_c(), 8, *_c(), N, 0.1, out=_t(1, 4, 32)),
    "workspace": lambda: cmc.cmc_two_tier_decode_q4(Q, *_c(), 8, *_c(), N, 0.1, workspace=_t(64, 2)[:, 0]),
    "rope: nothing": lambda: cmc.cmc_norm_rope(None, None, None, POS, F),
    "rope: v alone": lambda: cmc.cmc_norm_rope(X, None, X, POS, F),
    "rope: pos": lambda: cmc.cmc_norm_rope(X, X, X, POS.long(), F),
    "rope: pos' shape": lambda: cmc.cmc_norm_rope(X, X, X, POS[:1].contiguous(), F),
    "rope: frequencies": lambda: cmc.cmc_norm_rope(X, X, X, POS, F.double()),
    "rope: weight": lambda: cmc.cmc_norm_rope(X, X, X, POS, F, q_weight=_t(32)),
    "rope: types": lambda: cmc.cmc_norm_rope(X, X.bfloat16(), X.bfloat16(), POS, F),
    "rope: heads": lambda: cmc.cmc_norm_rope(X, X, X[:, :, :2], POS, F),
    "rope: strided heads": lambda: cmc.cmc_norm_rope(_t(2, 3, 4, 128)[..., :64], None, None, POS, F),
    "rope: uneven tokens": lambda: cmc.cmc_norm_rope(_t(2, 5, 4, 64)[:, :3], None, None, POS, F),
    "rope: out_q": lambda: cmc.cmc_norm_rope(X, None, None, POS, F, out_q=_t(2, 4, 3, 64)),
    "rope: out_k": lambda: cmc.cmc_norm_rope(None, X, None, POS, F, out_k=_t(2, 3, 4, 64)),
    "rope: 3-d": lambda: cmc.cmc_norm_rope(X[0], None, None, POS, F),
}


@pytest.fixture
def on_host(monkeypatch):
    """The wrappers' own checks, which come before anything needs a GPU."""
    monkeypatch.setattr(cmc, "_torch", torch)
    monkeypatch.setattr(cmc, "_device_index", lambda: -1)


@pytest.mark.parametrize("what", sorted(WRAPPER_REFUSALS))
def test_wrapper_refusals(on_host, what):
    with pytest.raises((ValueError, TypeError)):
        WRAPPER_REFUSALS[what]()


def test_host_tensors_are_refused(monkeypatch):
    monkeypatch.setattr(cmc, "_torch", torch)
    monkeypatch.setattr(cmc, "_device_index", lambda: 0)
    for call in (lambda: cmc.cmc_window_append_q4(*_c(), N, NEW, NEW), lambda: cmc.cmc_cache_read_q4(*_c()),
                 lambda: cmc.cmc_two_tier_decode_q4(Q, *_c(), 8, *_c(), N, 0.1),
                 lambda: cmc.cmc_gather_tier1_q4(_t(1, 2, 8, 64), _t(1, 2, 8, 64), None, 4),
                 lambda: cmc.cmc_norm_rope(X, X, X, POS, F)):
        with pytest.raises(ValueError, match="takes device tensors"):
            call()


C8, POOL = _c(), _t(1, 2, 50, 64)
# Every wrapper, and how many tensors it makes.
MAKES = {
    "gather": (4, lambda s: cmc.cmc_gather_tier1_q4(POOL, POOL, None, 8, stream=s)),
    "read": (2, lambda s: cmc.cmc_cache_read_q4(*C8, stream=s)),
    "decode": (2, lambda s: cmc.cmc_two_tier_decode_q4(Q, *C8, 8, *C8, N, 0.1, stream=s)),
    "step": (2, lambda s: cmc.cmc_decode_step_q4(Q, *C8, 8, *C8, N, NEW, NEW, 0.1, stream=s)),
    "append": (0, lambda s: cmc.cmc_window_append_q4(*C8, N, NEW, NEW, stream=s)),
    "rope": (3, lambda s: cmc.cmc_norm_rope(X, X, X, POS, F, stream=s)),
}


@pytest.mark.parametrize("name", sorted(MAKES))
def test_made_on_the_calls_stream(made, monkeypatch, name):  # noqa: F811
    monkeypatch.setattr(cmc, "_q4_calls", None)
    monkeypatch.setattr(cmc, "_rope_call", None)
    log, calls = made
    count, call = MAKES[name]
    side = Stream(4096)
    for stream, handle, where in ((None, 7, MAIN), (side, 4096, side), (4096, 4096, ("external", 4096)), (0, 0, "default")):
        log.clear()
        calls.clear()
        call(stream)
        assert len(log) == count and {w for _, w in log} <= {where}, (stream, log)
        assert [h for _, h in calls] == [handle], calls


def test_token_strides_of_slices(monkeypatch):
    """The parts of one projection go to the library as they lie."""
    seen = {}
    monkeypatch.setattr(cmc, "_torch", torch)
    monkeypatch.setattr(cmc, "_device_index", lambda: -1)
    monkeypatch.setattr(cmc, "_raw_stream", lambda d: 0)
    monkeypatch.setattr(cmc, "_rope_call", lambda *a: seen.update(a=a) and 0)
    x = _t(2, 3, 8, 64)
    q, k, v = x[:, :, :4], x[:, :, 4:6], x[:, :, 6:]
    cmc.cmc_norm_rope(q, k, v, POS, F)
    a = seen["a"]
    assert a[1] == a[3] == a[5] == 512 and a[2] - a[0] == 4 * 64 * 4 and a[4] - a[0] == 6 * 64 * 4
    one = _t(2, 1, 8, 64)
    cmc.cmc_norm_rope(one[:, :, :4], None, None, _t(2, 1, dtype=torch.int32), F)
    assert seen["a"][1] == 512 and seen["a"][2] is None
    single = _t(1, 1, 8, 64)
    cmc.cmc_norm_rope(single[:, :, :4], None, None, _t(1, 1, dtype=torch.int32), F)
    assert seen["a"][1] == 256


# ------------------------------------------------------------- the reference

def test_reference_rounding():
    """The nearest magnitude, by search; ties to the even code; scales by their two
    inequalities."""
    rng = np.random.default_rng(0)
    y = np.concatenate([rng.uniform(-6, 6, 4000), q4_ref.MAGNITUDES, [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]])
    c = q4_ref.round_code(y)
    got = q4_ref.MAGNITUDES[c & 7]
    off = np.abs(np.abs(y)[:, None] - q4_ref.MAGNITUDES)
    assert (np.abs(np.abs(y) - got) == off.min(axis=1)).all()
    ties = (off == off.min(axis=1, keepdims=True)).sum(axis=1) == 2
    assert ties.sum() == 7 and (c[ties] % 2 == 0).all()
    assert ((c >= 8) == np.signbit(y)).all()
    for e in range(-130, 128):
        for m in (1.0, 1.4999999, 1.5, 1.5000001, 1.9999999):
            a = np.float32(np.ldexp(m, e))
            if np.isfinite(a):
                s = q4_ref.scale_byte([float(a), 0.0, -np.inf])
                assert s >= 1 and float(a) <= 6 * 2.0 ** (s - 127) and (s == 1 or float(a) > 6 * 2.0 ** (s - 128))
    assert q4_ref.scale_byte([0.0]) == 1 and q4_ref.scale_byte([np.inf]) == 1 and q4_ref.scale_byte([1.0, np.nan]) == 255


def test_reference_pack():
    c = np.arange(16)
    assert (q4_ref.unpack(q4_ref.pack(c)) == c).all()
    assert q4_ref.pack(np.array([1, 2])).tolist() == [0x21]
    assert q4_ref.newest(5, 3, 5) == [0, 1, 2] and q4_ref.newest(5, 7, 2) == [0, 1] and q4_ref.newest(5, 5, 2) == [3, 4]
    assert q4_ref.newest(5, 12, 9) == [2, 3, 4, 0, 1] and q4_ref.newest(5, -1, 3) == []
