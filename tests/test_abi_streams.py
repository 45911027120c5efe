"""Calls on a stream that is not the current one: what a wrapper makes itself
(outputs, workspaces and their zero fill) is made on that stream.  On the CPU,
with the library's calls and torch's stream context replaced by recorders."""
import contextlib

import pytest
import torch

from paper_2609_25537_amd import cmc

MAIN = "the current stream"


class Stream:
    """A stand-in for a torch stream."""

    def __init__(self, handle):
        self.cuda_stream = handle


@pytest.fixture
def made(monkeypatch):
    """Records, for each tensor that a wrapper makes, the stream it is made on;
    and the stream handle that each library call gets."""
    on, log, calls = [MAIN], [], []

    @contextlib.contextmanager
    def context(stream):
        on.append(stream)
        yield
        on.pop()

    def recorded(name):
        real = getattr(torch, name)

        def make(*a, **kw):
            log.append((name, on[-1]))
            return real(*a, **kw)
        monkeypatch.setattr(torch, name, make)

    for name in ("empty", "zeros", "empty_like"):
        recorded(name)
    monkeypatch.setattr(torch.cuda, "stream", context)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda h: ("external", h))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda: "default")

    real = cmc.lib()

    class Library:
        """The C calls as recorders; the size queries are the library's."""

        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return getattr(real, name)

            def call(*a):
                calls.append((name, a[-1]))
                return 0
            return call

    library = Library()
    monkeypatch.setattr(cmc, "lib", lambda: library)
    monkeypatch.setattr(cmc, "_q8_calls", None)
    monkeypatch.setattr(cmc, "_torch", torch)
    monkeypatch.setattr(cmc, "_device_index", lambda: -1)  # what get_device() gives for a host tensor
    monkeypatch.setattr(cmc, "_raw_stream", lambda d: 7)
    monkeypatch.setattr(cmc, "_ptr", lambda t: None if t is None else t.data_ptr())
    yield log, calls
    cmc._q8_calls = None


f32, i32, bf16, e4 = torch.float32, torch.int32, torch.bfloat16, torch.float8_e4m3fn


def _z(*shape, dtype=f32):
    return torch.ones(shape, dtype=f32).mul(0).to(dtype)


def _decode():
    q, pool, win, new = _z(1, 4, 64), _z(1, 2, 50, 64), _z(1, 2, 40, 64), _z(1, 2, 1, 64)
    return q, pool, win, new, _z(1, dtype=i32)


def _q8(R=40):
    return [_z(1, 2, R, 64, dtype=e4), _z(1, 2, R, 64, dtype=e4), _z(1, 2, 2), _z(1, 2, 2)]


def _calls():
    """Every wrapper that makes something, and how many tensors it makes."""
    q, pool, win, new, n = _decode()
    idx = _z(1, 8, dtype=i32)
    emb = _z(1, 32, 64)
    h, w1, w2, b = _z(3, 64, dtype=bf16), _z(128, 64, dtype=bf16), _z(64, 128, dtype=bf16), _z(64)
    return {
        "select": (2, lambda s: cmc.cmc_select_cmes(_z(1, 50, 64), _z(1, 64), 8, stream=s)),
        "select_ragged": (3, lambda s: cmc.cmc_select_cmes_ragged(_z(1, 50, 64), _z(1, 64), n, 8, stream=s)),
        "locate": (2, lambda s: cmc.cmc_locate_window(_z(1, 50), n, 16, 4, stream=s)),
        "bridge": (2, lambda s: cmc.cmc_memory_bridge(h, w1, _z(128), w2, b, b, b, 0.1, stream=s)),
        "denoise": (5, lambda s: cmc.cmc_denoise(emb, chunk_tokens=8, stream=s)),
        "gather": (2, lambda s: cmc.cmc_gather_tier1(pool, pool, idx, 8, stream=s)),
        "decode": (2, lambda s: cmc.cmc_two_tier_decode(q, pool, pool, None, 8, win, win, n, 0.1, stream=s)),
        "step": (2, lambda s: cmc.cmc_decode_step(q, pool, pool, None, 8, win, win, n, new, new, 0.1, stream=s)),
        "decode_ragged": (2, lambda s: cmc.cmc_two_tier_decode_ragged(q, pool, pool, idx, n, 8, win, win, n, 0.1,
                                                                       stream=s)),
        "step_ragged": (2, lambda s: cmc.cmc_decode_step_ragged(q, pool, pool, idx, n, 8, win, win, n, new, new, 0.1,
                                                                 stream=s)),
        "step_noalloc": (1, lambda s: cmc.cmc_decode_step_noalloc(q, pool, pool, idx, 8, win, win, n, new, new, 0.1,
                                                                   stream=s)),
        "gather_q8": (4, lambda s: cmc.cmc_gather_tier1_q8(pool, pool, None, 8, 32, stream=s)),
        "read_q8": (2, lambda s: cmc.cmc_cache_read_q8(*_q8(), 32, stream=s)),
        "decode_q8": (2, lambda s: cmc.cmc_two_tier_decode_q8(q, *_q8(), 40, *_q8(), n, 0.1, 32, stream=s)),
        "step_q8": (2, lambda s: cmc.cmc_decode_step_q8(q, *_q8(), 40, *_q8(), n, new, new, 0.1, 32, stream=s)),
    }


NAMES = ["select", "select_ragged", "locate", "bridge", "denoise", "gather", "decode", "step", "decode_ragged", "step_ragged",
         "step_noalloc", "gather_q8", "read_q8", "decode_q8", "step_q8"]


@pytest.mark.parametrize("name", NAMES)
def test_made_on_the_calls_stream(made, name):
    log, calls = made
    count, call = _calls()[name]
    side = Stream(4096)
    for stream, handle, where in ((None, 7, MAIN), (side, 4096, side), (4096, 4096, ("external", 4096)), (0, 0, "default")):
        log.clear()
        calls.clear()
        call(stream)
        assert len(log) == count and {w for _, w in log} == {where}, (stream, log)
        assert [h for _, h in calls] == [handle], calls


def test_every_wrapper_that_makes_something_is_here():
    assert sorted(NAMES) == sorted(_calls())
