"""Memory that a call makes for work on another stream comes from that stream (no GPU needed: the
library's entry points are replaced, and tensors on the CPU stand for those of the device).

The caching allocator hands a freed block out again at once on the stream that it belongs to.  A
block of the current stream may so still be in use by work pending there, which a launch on another
stream does not wait for."""
import contextlib

import pytest
import torch


class Stream:
    def __init__(self, cuda_stream):
        self.cuda_stream = cuda_stream


CURRENT, SIDE = Stream(0), Stream(77)


class Allocations:
    """Which stream every tensor was made on, and on which streams its use was recorded."""

    def __init__(self):
        self.stack, self.made, self.recorded = [CURRENT], [], {}

    def stream_of(self, t):
        return [s for p, s in self.made if p == t.data_ptr()]


@pytest.fixture
def sp(monkeypatch):
    from paper_2501_16376_b200 import binding
    real = binding.lib
    log = Allocations()

    class Library:
        def __getattr__(self, name):
            if name in ("sp_mx4_scale_bytes", "sp_mx4_linear_workspace", "sp_cache_attention_workspace", "sp_status_string"):
                return getattr(real, name)
            return lambda *a: binding.SP_OK

    def noting(make):
        def made(*a, **kw):
            t = make(*a, **kw)
            log.made.append((t.data_ptr(), log.stack[-1]))
            log.keep.append(t)
            return t
        return made
    log.keep = []

    @contextlib.contextmanager
    def scope(stream):
        log.stack.append(stream)
        yield
        log.stack.pop()

    def matrix(t, what, host=False):
        return t.data_ptr(), t.shape[0], t.shape[1], t.stride(0)
    monkeypatch.setattr(binding, "lib", Library())
    monkeypatch.setattr(binding, "_matrix", matrix)
    monkeypatch.setattr(binding, "_current_device", lambda: -1)
    monkeypatch.setattr(torch.cuda, "stream", scope)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: log.stack[-1])
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: CURRENT)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda p, device=None: {77: SIDE}[p])
    monkeypatch.setattr(torch.Tensor, "record_stream",
                        lambda t, s: log.recorded.setdefault(t.data_ptr(), []).append(s))
    for name in ("empty", "empty_like", "zeros"):
        monkeypatch.setattr(torch, name, noting(getattr(torch, name)))
    monkeypatch.setattr(binding, "log", log, raising=False)
    return binding


def _cache(sp, blocks=4):
    k, v = (torch.full((blocks, 2, 16, 64), 1, dtype=torch.uint8) for _ in range(2))
    ks, vs = (torch.ones(blocks, 2) for _ in range(2))
    return sp.KvCache(k, v, ks, vs, torch.arange(blocks, dtype=torch.int32).view(2, -1))


def _quantize(sp, stream):
    return sp.sp_mx4_quantize(torch.ones(64, 64, dtype=torch.float16), stream=stream)


def _dequantize(sp, stream):
    return sp.sp_mx4_dequantize(torch.full((64, 32), 1, dtype=torch.uint8), torch.full((512,), 1, dtype=torch.uint8), 64, stream=stream),


def _linear(sp, stream):
    return sp.sp_mx4_linear(torch.ones(300, 64, dtype=torch.float16), torch.full((64, 32), 1, dtype=torch.uint8),
                            torch.full((512,), 1, dtype=torch.uint8), sp.SP_MX4_A4, stream=stream),


def _attention(sp, stream):
    acc = torch.ones(2, 2, 32)
    return _cache(sp).sp_cache_attention(torch.ones(2, 1, 4, 64, dtype=torch.float16), torch.ones(2, dtype=torch.int32), 32,
                                         acc_in=acc, acc_out=acc, stream=stream),


def _evict(sp, stream):
    return _cache(sp).sp_cache_evict(torch.ones(2, dtype=torch.int32), 32, torch.ones(2, 2, 32), 16, 4, _cache(sp),
                                     stream=stream)


SERVING = [_quantize, _dequantize, _linear, _attention, _evict]


def _check(sp, call, stream):
    log = sp.log
    outs = call(sp, stream)
    assert log.made and all(s is SIDE for _, s in log.made), [s.cuda_stream for _, s in log.made]
    for t in outs:                                    # the caller goes on using these where it is
        assert CURRENT in log.recorded.get(t.data_ptr(), [])


@pytest.mark.parametrize("stream", [SIDE, 77])
@pytest.mark.parametrize("call", SERVING)
def test_serving_calls_allocate_on_the_stream_they_work_on(sp, call, stream):
    _check(sp, call, stream)


@pytest.mark.parametrize("call", SERVING)
def test_the_default_stream_may_be_named_by_its_handle(sp, call):
    call(sp, 0)
    assert sp.log.made and all(s is CURRENT for _, s in sp.log.made)


def _context(sp):
    ctx = sp.Context.__new__(sp.Context)
    ctx.d_in, ctx._h = 64, None
    return ctx


def _W():
    return torch.ones(16, 64, dtype=torch.float16)


PRUNING = [
    lambda sp, s: [_context(sp).sp_score(_W(), stream=s)],
    lambda sp, s: _context(sp).sp_select_24_compressed(_W(), stream=s),
    lambda sp, s: _context(sp).sp_select_unstructured(_W(), 0.5, stream=s),
    lambda sp, s: _context(sp).sp_select_nm(_W(), 2, 4, stream=s),
    lambda sp, s: _context(sp).sp_ewma_trace(_W(), sp.EwmaParams(0.1, 0.1, 1.0, 0), stream=s),
    lambda sp, s: sum(_context(sp).sp_select_unstructured_group([_W(), _W()], 0.5, stream=s), []),
    lambda sp, s: sum(_context(sp).sp_select_nm_group([_W(), _W()], 2, 4, stream=s), []),
    lambda sp, s: sum(sp.sp_select_unstructured_multi([_context(sp)], [_W()], 0.5, stream=s), []),
    lambda sp, s: sum(sp.sp_select_nm_multi([_context(sp)], [_W()], 2, 4, stream=s), []),
    lambda sp, s: [sp.sp_apply_mask(_W(), torch.ones(16, 2, dtype=torch.int32), stream=s)],
]


@pytest.mark.parametrize("call", PRUNING)
def test_pruning_calls_allocate_on_the_stream_they_work_on(sp, call):
    _check(sp, call, SIDE)
