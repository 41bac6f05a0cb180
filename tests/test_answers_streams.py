"""What the calls for several answers of one prompt make themselves comes from the stream that they work
on (no GPU needed: the library's entry points are replaced)."""
import pytest
import torch

from .test_serve_streams import CURRENT, SIDE, sp  # noqa: F401


@pytest.fixture
def calls(sp, monkeypatch):
    from paper_2501_16376_b200 import binding
    real, names = binding.lib, []

    class Library:
        def __getattr__(self, name):
            if name.endswith("_workspace"):
                return lambda c, *a: setattr(a[-1]._obj, "value", 4096) or 0
            return lambda *a: names.append((name, a[-1])) or 0
    monkeypatch.setattr(binding, "lib", Library())
    monkeypatch.setattr(binding, "_raw_stream", lambda stream, device: 0 if stream is None else stream.cuda_stream)
    return names


def _cache(sp):
    k, v = (torch.full((4, 2, 16, 64), 1, dtype=torch.uint8) for _ in range(2))
    ks, vs = (torch.ones(4, 2) for _ in range(2))
    return sp.KvCache(k, v, ks, vs, torch.arange(4, dtype=torch.int32).view(2, 2), refs=torch.ones(4, dtype=torch.int32))


def _rotary(sp, stream):
    Q = torch.ones(2, 1, 4, 64, dtype=torch.float16)
    return sp.sp_qk_norm_rotary(Q, Q, torch.ones(2, dtype=torch.int32), torch.ones(32), stream=stream)


def _fork(sp, stream):
    _cache(sp).sp_cache_fork(torch.ones(2, dtype=torch.int32), stream=stream)
    return ()


def _reserve(sp, stream):
    return _cache(sp).sp_cache_reserve(torch.ones(2, dtype=torch.int32), 3, stream=stream),


def _compact(sp, stream):
    return _cache(sp).sp_cache_compact(stream=stream),


def _shared(sp, stream):
    return _cache(sp).sp_cache_attention_shared(torch.ones(2, 1, 4, 64, dtype=torch.float16), torch.ones(2, dtype=torch.int32), 32,
                                                torch.tensor([0, 2], dtype=torch.int32), torch.ones(1, dtype=torch.int32), 16, 2, stream=stream),


@pytest.mark.parametrize("call", [_rotary, _fork, _reserve, _compact, _shared])
def test_memory_of_the_stream(sp, calls, call):
    for stream in (None, SIDE):
        log = sp.log
        del log.made[:], log.keep[:]
        log.recorded.clear()
        outs = call(sp, stream)
        there = CURRENT if stream is None else SIDE
        made = [(p, s) for p, s in log.made if p]
        assert made and all(s is there for _, s in made[-(1 + len(outs)):])
        assert calls[-1][1] == there.cuda_stream
        for t in outs:                                      # results are also the caller's stream's
            assert (CURRENT in log.recorded.get(t.data_ptr(), [])) == (stream is not None)
