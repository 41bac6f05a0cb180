"""The calls for several answers of one prompt refuse bad arguments on the host, before anything is
launched (no GPU needed: nothing below gets as far as a launch)."""
import ctypes

import pytest
import torch

from .test_serve_devices import On0, On1, _t, sp  # noqa: F401
from .test_serve_refusals import P, _cache, b  # noqa: F401


def test_rotary(b):
    s = b.Strides(64, 64, 64)

    def call(Q=P, qs=s, H=2, K=P, ks=s, Hk=1, dtype=0, B=1, n=1, dim=64, w=None, eps=1e-6, start=P, freq=P, rotary=64, Qo=P, Ko=P, os=s):
        return b.lib.sp_qk_norm_rotary(Q, qs, H, K, ks, Hk, dtype, B, n, dim, w, w, eps, start, freq, rotary, 0, Qo, os, Ko, os, None)
    assert call(dtype=4) == b.SP_ERR_DTYPE
    for kw in (dict(dim=0), dict(dim=63), dict(dim=258, rotary=2), dict(rotary=66), dict(rotary=-2), dict(rotary=3),
               dict(H=65535), dict(B=1 << 20, n=1 << 20)):
        assert call(**kw) == b.SP_ERR_SHAPE, kw
    for kw in (dict(H=-1), dict(Hk=-1), dict(B=-1), dict(n=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(Q=None), dict(K=None),
               dict(Qo=None), dict(Ko=None), dict(qs=None), dict(os=None), dict(start=None), dict(freq=None)):
        assert call(**kw) == b.SP_ERR_INVALID_ARG, kw
    assert call(B=0, Q=None, K=None) == b.SP_OK and call(n=0) == b.SP_OK and call(H=0, Hk=0, Q=None) == b.SP_OK


@pytest.mark.parametrize("kw", [dict(head_dim=96), dict(n_blocks=1 << 31), dict(ld_table=3)])
def test_pages_of_a_bad_cache(b, kw):
    c, n = _cache(b, **kw), ctypes.c_int64()
    assert b.lib.sp_cache_fork(c, P, P, P, 1, None, 0, None) == b.SP_ERR_SHAPE
    assert b.lib.sp_cache_reserve(c, P, P, P, 1, P, P, 1 << 40, None) == b.SP_ERR_SHAPE
    assert b.lib.sp_cache_compact(c, P, P, 4, P, P, P, 1 << 40, None) == b.SP_ERR_SHAPE
    assert b.lib.sp_cache_compact_workspace(c, ctypes.byref(n)) == b.SP_ERR_SHAPE


def test_pages(b):
    c, n = _cache(b), ctypes.c_int64()
    fork = lambda refs=P, dst=P, n=1, ws=P, c=c: b.lib.sp_cache_fork(c, refs, dst, None, n, ws, 1 << 40 if ws else 0, None)
    assert fork(refs=None) == b.SP_ERR_INVALID_ARG and fork(dst=None) == b.SP_ERR_INVALID_ARG and fork(n=-1) == b.SP_ERR_INVALID_ARG
    assert fork(n=1 << 30) == b.SP_ERR_SHAPE and fork(n=0, refs=None, dst=None) == b.SP_OK
    assert fork(n=100000, ws=None) == b.SP_ERR_INVALID_ARG and fork(n=100000, ws=P + 8) == b.SP_ERR_INVALID_ARG
    reserve = lambda refs=P, start=P, n=1, status=P, ws=P, size=1 << 40: b.lib.sp_cache_reserve(c, refs, start, None, n, status, ws, size, None)
    for kw in (dict(refs=None), dict(start=None), dict(n=-1), dict(status=None), dict(ws=None), dict(ws=P + 4), dict(size=16)):
        assert reserve(**kw) == b.SP_ERR_INVALID_ARG, kw
    assert reserve(n=1 << 40) == b.SP_ERR_SHAPE
    wide = _cache(b, n_seqs=32767, table_cols=1 << 20, ld_table=1 << 20)
    assert b.lib.sp_cache_reserve_workspace(wide, 1 << 29, ctypes.byref(n)) == b.SP_ERR_SHAPE
    compact = lambda refs=P, table=2 * P, ld=4, out=P, live=P, ws=P, size=1 << 40: b.lib.sp_cache_compact(c, refs, table, ld, out, live, ws, size, None)
    for kw in (dict(refs=None), dict(table=None), dict(out=None), dict(live=None), dict(ws=None), dict(ws=P + 4), dict(size=16)):
        assert compact(**kw) == b.SP_ERR_INVALID_ARG, kw
    assert compact(ld=3) == b.SP_ERR_SHAPE and compact(table=P, ld=5) == b.SP_ERR_SHAPE


def test_shared_attention(b):
    c, s, n = _cache(b), b.Strides(64, 64, 64), ctypes.c_int64()

    def call(Q=P, dtype=0, n_q=1, heads=4, lens=P, max_len=64, starts=P, groups=1, prefix=P, max_prefix=32, max_group=2, scale=0.1, O=P,
             ws=P, size=1 << 40, c=c):
        return b.lib.sp_cache_attention_shared(c, Q, s, dtype, n_q, heads, lens, max_len, starts, groups, prefix, max_prefix, max_group,
                                               scale, O, s, None, ws, size, None)
    assert call(dtype=3) == b.SP_ERR_DTYPE
    for kw in (dict(heads=3), dict(n_q=100000), dict(max_len=1 << 40), dict(groups=40000), dict(max_prefix=1 << 40), dict(max_group=40000),
               dict(c=_cache(b, n_blocks=1 << 31))):
        assert call(**kw) == b.SP_ERR_SHAPE, kw
    for kw in (dict(heads=0), dict(n_q=-1), dict(max_len=-1), dict(groups=-1), dict(max_prefix=-1), dict(max_group=-1), dict(scale=float("inf")),
               dict(Q=None), dict(O=None), dict(lens=None), dict(starts=None), dict(prefix=None)):
        assert call(**kw) == b.SP_ERR_INVALID_ARG, kw
    many = _cache(b, n_seqs=32767, n_kv_heads=512, head_dim=128)
    assert call(c=many, n_q=1, heads=4096, max_group=32767) == b.SP_ERR_SHAPE      # 1024 tiles of rows for 512 heads
    assert b.lib.sp_cache_attention_shared_workspace(c, 1, 4, 64, 1, 32, 2, ctypes.byref(n)) == b.SP_OK
    if n.value:
        assert call(ws=None) == b.SP_ERR_INVALID_ARG and call(size=n.value - 1) == b.SP_ERR_INVALID_ARG
    assert call(n_q=0, Q=None, O=None, lens=None) == b.SP_OK


def _handle(sp, on, device, refs=True):
    sp.at(device)
    u8, f32, i32 = dict(dtype=torch.uint8), dict(dtype=torch.float32), dict(dtype=torch.int32)
    return sp.KvCache(_t(on, 4, 2, 16, 64, **u8), _t(on, 4, 2, 16, 64, **u8), _t(on, 4, 2, **f32), _t(on, 4, 2, **f32),
                      torch.arange(4, dtype=torch.int32).view(2, 2).as_subclass(on), refs=_t(on, 4, **i32) if refs else None)


def test_another_device_and_a_cache_without_counts(sp):
    i32 = dict(dtype=torch.int32)
    for cache, device, on, good in ((_handle(sp, On0, 0), 0, On0, True), (_handle(sp, On0, 0), 1, On1, False),
                                    (_handle(sp, On0, 0), 0, On1, False), (_handle(sp, On0, 0, refs=False), 0, On0, False)):
        sp.at(device)
        n, ws = _t(on, 2, **i32), _t(on, 1 << 20, dtype=torch.uint8)
        for call in (lambda: cache.sp_cache_fork(n, n), lambda: cache.sp_cache_reserve(n, 3, status=n, workspace=ws),
                     lambda: cache.sp_cache_compact(_t(on, 1, **i32), workspace=ws)):
            del sp.calls[:]
            if good:
                call()
                assert len(sp.calls) == 1
            else:
                with pytest.raises(sp.SpError):
                    call()
                assert not sp.calls
    sp.at(0)
    with pytest.raises(sp.SpError):                          # refs of another device, or size
        c = _handle(sp, On0, 0)
        sp.KvCache(c.k, c.v, c.k_scale, c.v_scale, c.table, refs=_t(On1, 4, **i32))
    with pytest.raises(sp.SpError):
        sp.KvCache(c.k, c.v, c.k_scale, c.v_scale, c.table, refs=_t(On0, 5, **i32))


def test_shared_attention_checks_its_tensors(sp):
    i32, cache = dict(dtype=torch.int32), _handle(sp, On0, 0, refs=False)
    good = dict(Q=_t(On0, 2, 1, 4, 64), lens=_t(On0, 2, **i32), max_len=32, group_start=_t(On0, 2, **i32), prefix=_t(On0, 1, **i32),
                max_prefix=16, max_group=2, O=_t(On0, 2, 1, 4, 64), workspace=_t(On0, 1 << 20, dtype=torch.uint8))
    cache.sp_cache_attention_shared(**good)
    assert sp.calls == ["sp_cache_attention_shared"]
    for kw in (dict(Q=_t(On1, 2, 1, 4, 64)), dict(Q=_t(On0, 3, 1, 4, 64)), dict(O=_t(On0, 2, 1, 4, 64, dtype=torch.bfloat16)),
               dict(O=good["Q"]), dict(lens=_t(On0, 3, **i32)), dict(group_start=_t(On0, 1, **i32)), dict(prefix=_t(On0, 2, **i32)),
               dict(prefix=_t(On1, 1, **i32)), dict(lse=_t(On0, 2, 1, 4)), dict(Q=_t(On0, 2, 1, 3, 64), O=_t(On0, 2, 1, 3, 64)),
               dict(workspace=_t(On1, 1 << 20, dtype=torch.uint8))):
        del sp.calls[:]
        if "workspace" in kw and cache.sp_cache_attention_shared(**good) is not None and not cache._need(
                "sp_cache_attention_shared_workspace", 1, 4, 32, 1, 16, 2):
            continue
        del sp.calls[:]
        with pytest.raises(sp.SpError):
            cache.sp_cache_attention_shared(**{**good, **kw})
        assert not sp.calls, kw


def test_rotary_checks_its_tensors(sp):
    sp.at(0)
    x = torch.ones(2, 3, 4, 64, dtype=torch.float16).as_subclass(On0)
    good = dict(Q=x, K=_t(On0, 2, 3, 2, 64), start=_t(On0, 2, dtype=torch.int32), freq=_t(On0, 32, dtype=torch.float32),
                Q_out=_t(On0, 2, 3, 4, 64), K_out=_t(On0, 2, 3, 2, 64))
    sp.sp_qk_norm_rotary(**good)
    sp.sp_qk_norm_rotary(**{**good, "Q_out": x})
    assert sp.calls == ["sp_qk_norm_rotary"] * 2
    for kw in (dict(Q=_t(On1, 2, 3, 4, 64)), dict(K=_t(On0, 2, 4, 2, 64)), dict(K=_t(On0, 2, 3, 2, 32)), dict(K_out=_t(On0, 2, 3, 4, 64)),
               dict(Q_out=_t(On0, 2, 3, 4, 64, dtype=torch.bfloat16)), dict(start=_t(On0, 3, dtype=torch.int32)),
               dict(start=_t(On0, 2, dtype=torch.int64)), dict(freq=_t(On0, 32)), dict(freq=_t(On0, 33, dtype=torch.float32)[:, None]),
               dict(q_weight=_t(On0, 32)), dict(k_weight=_t(On0, 64, dtype=torch.float32)), dict(k_weight=_t(On1, 64)),
               dict(Q_out=x.as_strided(x.shape, (768, 64, 192, 1)))):
        del sp.calls[:]
        with pytest.raises(sp.SpError):
            sp.sp_qk_norm_rotary(**{**good, **kw})
        assert not sp.calls, kw
