"""Serving calls refuse memory of a device that is not the current one (no GPU needed: the library's
entry points are replaced, and CPU tensors stand for those of devices 0 and 1)."""
import pytest
import torch


class On0(torch.Tensor):
    def get_device(self):
        return 0


class On1(torch.Tensor):
    def get_device(self):
        return 1


@pytest.fixture
def sp(monkeypatch):
    from paper_2501_16376_b200 import binding
    real, calls = binding.lib, []

    class Library:
        def __getattr__(self, name):
            if name.endswith("_workspace") or name in ("sp_mx4_scale_bytes", "sp_status_string"):
                return getattr(real, name)
            return lambda *a: calls.append(name) or binding.SP_OK
    monkeypatch.setattr(binding, "lib", Library())
    monkeypatch.setattr(binding, "_raw_stream", lambda stream, device: 0)
    monkeypatch.setattr(binding, "calls", calls, raising=False)
    monkeypatch.setattr(binding, "at", lambda d: monkeypatch.setattr(binding, "_current_device", lambda: d), raising=False)
    return binding


def _t(on, *shape, dtype=torch.float16):
    return torch.ones(*shape, dtype=dtype).as_subclass(on)


def _cache(sp, on, device):
    sp.at(device)
    u8, f32 = dict(dtype=torch.uint8), dict(dtype=torch.float32)
    return sp.KvCache(_t(on, 4, 2, 16, 64, **u8), _t(on, 4, 2, 16, 64, **u8), _t(on, 4, 2, **f32), _t(on, 4, 2, **f32),
                      torch.arange(4, dtype=torch.int32).view(2, 2).as_subclass(on))


def test_a_cache_is_used_on_its_own_device_only(sp):
    cache = _cache(sp, On0, 0)
    for device, on in ((0, On0), (1, On1)):
        sp.at(device)
        x, n = _t(on, 2, 1, 2, 64), _t(on, 2, dtype=torch.int32)
        acc, i32 = _t(on, 2, 2, 32, dtype=torch.float32), dict(dtype=torch.int32)
        calls = [lambda: cache.sp_cache_append(x, x, n), lambda: cache.sp_cache_attention(x, n, 32, O=_t(on, 2, 1, 2, 64))]
        for dst in (_cache(sp, On0, 0), _cache(sp, On1, 1)):
            calls.append(lambda dst=dst: cache.sp_cache_evict(
                n, 32, acc, 16, 4, dst, acc_out=_t(on, 2, 2, 16, dtype=torch.float32), kept_out=_t(on, 2, 2, 16, **i32),
                lens_out=_t(on, 2, **i32)))
        sp.at(device)
        for i, call in enumerate(calls):
            del sp.calls[:]
            if device == 0 and i < 3:                   # the last one evicts into a cache of device 1
                call()
                assert len(sp.calls) == 1
            else:
                with pytest.raises(sp.SpError):
                    call()
                assert not sp.calls


def test_a_workspace_of_another_device(sp):
    sp.at(0)
    u8 = dict(dtype=torch.uint8)
    X, codes, scales = _t(On0, 300, 64), _t(On0, 64, 32, **u8), _t(On0, 512, **u8)
    call = lambda on: sp.sp_mx4_linear(X, codes, scales, sp.SP_MX4_A4, Y=_t(On0, 300, 64),
                                       workspace=_t(on, 1 << 20, **u8))
    call(On0)
    assert sp.calls == ["sp_mx4_linear"]
    with pytest.raises(sp.SpError):
        call(On1)
    cache = _cache(sp, On0, 0)
    acc = _t(On0, 2, 2, 32, dtype=torch.float32)
    attend = lambda on: cache.sp_cache_attention(_t(On0, 2, 1, 4, 64), _t(On0, 2, dtype=torch.int32), 32,
                                                 O=_t(On0, 2, 1, 4, 64), acc_out=acc, workspace=_t(on, 1 << 20, **u8))
    attend(On0)
    with pytest.raises(sp.SpError):
        attend(On1)
    assert sp.calls == ["sp_mx4_linear", "sp_cache_attention"]


def test_outputs_that_the_kernels_read_beside_writing_them(sp):
    """Kernels of one call read lens, acc and X in some blocks while others write the outputs."""
    src, dst = _cache(sp, On0, 0), _cache(sp, On0, 0)
    lens, acc = _t(On0, 2, dtype=torch.int32), _t(On0, 2, 2, 32, dtype=torch.float32)
    evict = lambda **kw: src.sp_cache_evict(lens, 32, acc, 32, 4, dst, **{
        **dict(kept_out=_t(On0, 2, 2, 32, dtype=torch.int32), acc_out=_t(On0, 2, 2, 32, dtype=torch.float32),
               lens_out=_t(On0, 2, dtype=torch.int32)), **kw})
    evict()
    for kw in (dict(lens_out=lens), dict(acc_out=acc)):
        with pytest.raises(sp.SpError):
            evict(**kw)
    X, codes, scales = _t(On0, 64, 64), _t(On0, 64, 32, dtype=torch.uint8), _t(On0, 512, dtype=torch.uint8)
    with pytest.raises(sp.SpError):
        sp.sp_mx4_linear(X, codes, scales, Y=X)
    assert sp.calls == ["sp_cache_evict"]
