"""The serving entry points refuse bad arguments on the host, before anything is launched (no GPU
needed: nothing below gets as far as a launch)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2501_16376_b200 import binding
    return binding


P = 4096  # stands for a device pointer; never dereferenced on the host


def test_scale_bytes(b):
    assert b.sp_mx4_scale_bytes(1, 1) == 512 and b.sp_mx4_scale_bytes(129, 129) == 4 * 512
    assert b.sp_mx4_scale_bytes(4096, 4096) == 4096 * 4096 // 32
    for rows, cols in ((0, 5), (5, 0), (-1, 5), (1, 1 << 40)):
        assert b.sp_mx4_scale_bytes(rows, cols) == 0


def test_quantize(b):
    q = b.lib.sp_mx4_quantize
    assert q(P, 7, 1, 32, 32, None, P, 16, P, None) == b.SP_ERR_DTYPE
    assert q(P, 0, -1, 32, 32, None, P, 16, P, None) == b.SP_ERR_INVALID_ARG
    assert q(P, 0, 1, 32, 31, None, P, 16, P, None) == b.SP_ERR_SHAPE
    assert q(P, 0, 1, 33, 33, None, P, 16, P, None) == b.SP_ERR_SHAPE       # codes too narrow
    assert q(P, 0, 1, 32, 32, None, P, 24, P, None) == b.SP_ERR_SHAPE
    assert q(P, 0, 1, 32, 32, None, P + 8, 16, P, None) == b.SP_ERR_INVALID_ARG
    assert q(P, 0, 1, 32, 32, None, None, 16, P, None) == b.SP_ERR_INVALID_ARG
    assert q(None, 0, 1, 32, 32, None, P, 16, P, None) == b.SP_ERR_INVALID_ARG
    assert q(None, 0, 0, 32, 32, None, None, 0, None, None) == b.SP_OK
    d = b.lib.sp_mx4_dequantize
    assert d(P, 16, P, 1, 32, 9, P, 32, None) == b.SP_ERR_DTYPE
    assert d(P, 16, P, 1, 32, 0, P, 31, None) == b.SP_ERR_SHAPE
    assert d(P, 16, P, 1, 32, 0, None, 32, None) == b.SP_ERR_INVALID_ARG


def test_linear(b):
    def call(X=P, dtype=1, T=2, ldx=64, codes=P, ldc=32, scales=P, rows=8, cols=64, mode=0, Y=P, ldy=8, ws=None, n=0):
        return b.lib.sp_mx4_linear(X, dtype, T, ldx, codes, ldc, scales, rows, cols, mode, Y, ldy, ws, n, None)
    assert call(dtype=2) == b.SP_ERR_DTYPE
    assert call(mode=2) == b.SP_ERR_INVALID_ARG and call(T=-1) == b.SP_ERR_INVALID_ARG
    assert call(cols=0, ldx=0) == b.SP_ERR_SHAPE and call(ldx=63) == b.SP_ERR_SHAPE and call(ldy=7) == b.SP_ERR_SHAPE
    assert call(ldc=16) == b.SP_ERR_SHAPE and call(ldc=40) == b.SP_ERR_SHAPE
    assert call(X=None) == b.SP_ERR_INVALID_ARG and call(Y=None) == b.SP_ERR_INVALID_ARG
    assert call(scales=P + 4) == b.SP_ERR_INVALID_ARG
    assert call(T=1 << 40) == b.SP_ERR_SHAPE
    assert call(T=0, X=None, Y=None) == b.SP_OK
    need = ctypes.c_int64()
    assert b.lib.sp_mx4_linear_workspace(1, 8, 64, 0, None) == b.SP_ERR_INVALID_ARG
    assert b.lib.sp_mx4_linear_workspace(1, 8, 64, 3, ctypes.byref(need)) == b.SP_ERR_INVALID_ARG
    assert b.lib.sp_mx4_linear_workspace(4096, 4096, 4096, 1, ctypes.byref(need)) == b.SP_OK
    if need.value:
        assert call(T=4096, ldx=4096, ldc=2048, rows=4096, cols=4096, ldy=4096, mode=1) == b.SP_ERR_INVALID_ARG


def _cache(b, **kw):
    f = dict(k=P, v=P, k_scale=P, v_scale=P, table=P, n_blocks=8, n_seqs=2, table_cols=4, ld_table=4, n_kv_heads=2,
             head_dim=64, block_tokens=16)
    f.update(kw)
    return b.CacheStruct(**f)


def test_cache_struct(b):
    s, n = b.Strides(64, 64, 64), ctypes.c_int64()
    for kw, want in ((dict(head_dim=96), b.SP_ERR_SHAPE), (dict(block_tokens=8), b.SP_ERR_SHAPE),
                     (dict(ld_table=3), b.SP_ERR_SHAPE), (dict(n_kv_heads=0), b.SP_ERR_INVALID_ARG),
                     (dict(n_kv_heads=70000), b.SP_ERR_SHAPE), (dict(n_seqs=70000), b.SP_ERR_SHAPE),
                     (dict(table=None), b.SP_ERR_INVALID_ARG), (dict(k=None), b.SP_ERR_INVALID_ARG),
                     (dict(v=P + 8), b.SP_ERR_INVALID_ARG), (dict(n_blocks=-1), b.SP_ERR_INVALID_ARG),
                     (dict(table_cols=1 << 40, ld_table=1 << 40), b.SP_ERR_SHAPE)):
        assert b.lib.sp_cache_append(_cache(b, **kw), P, s, P, s, 0, 1, P, None, None) == want, kw
        assert b.lib.sp_cache_attention_workspace(_cache(b, **kw), 1, 2, 64, 0, ctypes.byref(n)) == want, kw
    assert b.lib.sp_cache_append(None, P, s, P, s, 0, 1, P, None, None) == b.SP_ERR_INVALID_ARG


def test_append(b):
    c, s = _cache(b), b.Strides(64, 64, 64)
    assert b.lib.sp_cache_append(c, P, s, P, s, 5, 1, P, None, None) == b.SP_ERR_DTYPE
    assert b.lib.sp_cache_append(c, P, s, P, s, 0, -1, P, None, None) == b.SP_ERR_INVALID_ARG
    assert b.lib.sp_cache_append(c, P, None, P, s, 0, 1, P, None, None) == b.SP_ERR_INVALID_ARG
    assert b.lib.sp_cache_append(c, None, s, P, s, 0, 1, P, None, None) == b.SP_ERR_INVALID_ARG
    assert b.lib.sp_cache_append(c, P, s, P, s, 0, 1, None, None, None) == b.SP_ERR_INVALID_ARG
    assert b.lib.sp_cache_append(c, None, s, None, s, 0, 0, None, None, None) == b.SP_OK


def test_attention(b):
    c, s = _cache(b), b.Strides(64, 64, 64)

    def call(Q=P, dtype=0, n_q=1, heads=4, lens=P, max_len=64, scale=0.1, O=P, acc_out=None, ld=64, ws=P, n=1 << 40):
        return b.lib.sp_cache_attention(c, Q, s, dtype, n_q, heads, lens, max_len, scale, O, s, None, None, acc_out, ld,
                                        ws, n, None)
    assert call(dtype=3) == b.SP_ERR_DTYPE and call(heads=3) == b.SP_ERR_SHAPE and call(heads=0) == b.SP_ERR_INVALID_ARG
    assert call(n_q=-1) == b.SP_ERR_INVALID_ARG and call(n_q=100000) == b.SP_ERR_SHAPE
    assert call(max_len=-1) == b.SP_ERR_INVALID_ARG and call(max_len=1 << 40) == b.SP_ERR_SHAPE
    assert call(scale=float("inf")) == b.SP_ERR_INVALID_ARG
    assert call(Q=None) == b.SP_ERR_INVALID_ARG and call(lens=None) == b.SP_ERR_INVALID_ARG
    assert call(acc_out=P, ld=63) == b.SP_ERR_SHAPE
    assert call(acc_out=P, n=8) == b.SP_ERR_INVALID_ARG and call(acc_out=P, ws=None) == b.SP_ERR_INVALID_ARG
    assert call(n_q=0, Q=None, O=None, lens=None) == b.SP_OK


def test_evict(b):
    def call(src=None, dst=None, lens=P, max_len=64, acc=P, ld=64, budget=32, recent=4, kept=P, acc_out=P, ld_out=32):
        return b.lib.sp_cache_evict(src or _cache(b), lens, max_len, acc, ld, budget, recent, dst or _cache(b), kept,
                                    acc_out, ld_out, None, None)
    assert call(budget=-1) == b.SP_ERR_INVALID_ARG and call(recent=-1) == b.SP_ERR_INVALID_ARG
    assert call(dst=_cache(b, head_dim=128)) == b.SP_ERR_SHAPE and call(dst=_cache(b, n_seqs=3)) == b.SP_ERR_SHAPE
    assert call(dst=_cache(b, block_tokens=32)) == b.SP_ERR_SHAPE and call(dst=_cache(b, n_kv_heads=1)) == b.SP_ERR_SHAPE
    assert call(budget=65, ld_out=65) == b.SP_ERR_SHAPE                     # dst's table is too short
    assert call(ld=63) == b.SP_ERR_SHAPE and call(ld_out=31) == b.SP_ERR_SHAPE
    assert call(lens=None) == b.SP_ERR_INVALID_ARG and call(acc=None) == b.SP_ERR_INVALID_ARG
    assert call(kept=None) == b.SP_ERR_INVALID_ARG
    assert b.lib.sp_wait_status(None, 0) == b.SP_ERR_INVALID_ARG
