"""The 8-bit key/value cache against its definition in binary64."""
import numpy as np
import pytest
import torch

from . import serve_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = [torch.float16, torch.bfloat16]
UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def sp():
    from paper_2501_16376_b200 import binding
    return binding


def _cache(sp, n_seqs, tokens, heads, dim, block, seed=0, spare=2):
    """A cache whose blocks lie in a random order among spare ones, filled with stale bytes."""
    g = torch.Generator().manual_seed(seed)
    per = (tokens + block - 1) // block
    n = n_seqs * per + spare
    shape = (n, heads, block, dim)
    k, v = (torch.randint(0, 256, shape, generator=g, dtype=torch.uint8).cuda() for _ in range(2))
    ks, vs = (torch.exp2(torch.randint(-9, 9, shape[:2], generator=g).float()).cuda() for _ in range(2))
    table = torch.randperm(n, generator=g)[:n_seqs * per].view(n_seqs, per).to(torch.int32).cuda()
    return sp.KvCache(k, v, ks, vs, table)


def _kv(n_seqs, n, heads, dim, dtype, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(2, n_seqs, n, heads, dim, generator=g) * torch.exp(spread * torch.randn(2, n_seqs, n, 1, 1, generator=g))
    return x[0].to(dtype), x[1].to(dtype)


def _i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _same(cache, plain):
    for codes, want in ((cache.k, plain.k), (cache.v, plain.v)):
        got = codes.cpu().view(torch.float8_e4m3fn).double().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(np.nan_to_num(got), np.nan_to_num(want))
    for scale, e in ((cache.k_scale, plain.ke), (cache.v_scale, plain.ve)):
        assert np.array_equal(scale.cpu().double().numpy(), 2.0 ** e.astype(float))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,dim,block", [(1, 64, 16), (3, 128, 32), (2, 64, 64), (2, 128, 64), (5, 128, 16)])
def test_append_prompt_then_tokens(sp, heads, dim, block, dtype):
    cache = _cache(sp, 3, 200, heads, dim, block)
    plain = ref.PlainCache(cache)
    start = [0, 5, 17]
    for step, n in enumerate((70, 1, 1, 3, 40)):
        K, V = _kv(3, n, heads, dim, dtype, step)
        cache.sp_cache_append(K.cuda(), V.cuda(), _i32(*start))
        plain.append(K, V, start)
        _same(cache, plain)
        start = [s + n for s in start]


def test_append_ragged_counts_ends_of_the_table_and_absent_blocks(sp):
    heads, dim, block = 2, 64, 16
    cache = _cache(sp, 6, 64, heads, dim, block)
    cache.table[4, 1], cache.table[4, 2] = -1, 10 ** 6
    plain = ref.PlainCache(cache)
    K, V = _kv(6, 40, heads, dim, torch.float16, 1)
    start, count = [0, 30, 50, -3, 10, 63], [0, 7, 100, 5, 40, -2]
    cache.sp_cache_append(K.cuda(), V.cuda(), _i32(*start), _i32(*count))
    plain.append(K, V, start, count)
    _same(cache, plain)


def test_append_strided_and_unaligned_inputs(sp):
    cache = _cache(sp, 2, 64, 3, 64, 16)
    plain = ref.PlainCache(cache)
    g = torch.Generator().manual_seed(1)
    fused = torch.randn(2, 33, 3, 2, 65, generator=g).to(torch.bfloat16)
    K, V = fused[:, :, :, 0, 1:], fused[:, :, :, 1, :64]
    dev = fused.cuda()
    cache.sp_cache_append(dev[:, :, :, 0, 1:], dev[:, :, :, 1, :64], _i32(3, 20))
    plain.append(K, V, [3, 20])
    _same(cache, plain)


@pytest.mark.parametrize("dtype", DTYPES)
def test_append_special_values(sp, dtype):
    cache = _cache(sp, 1, 64, 1, 64, 16)
    plain = ref.PlainCache(cache)
    K, V = _kv(1, 48, 1, 64, dtype, 3)
    K[0, :16] = 0                                          # a block of zeros
    K[0, 20, 0, 5], K[0, 21, 0, 6], V[0, 3, 0, 1] = float("nan"), float("inf"), float("-inf")
    V[0, 16:32] = torch.finfo(dtype).tiny * 0.25
    V[0, 40] = torch.finfo(dtype).max
    cache.sp_cache_append(K.cuda(), V.cuda(), _i32(0))
    plain.append(K, V, [0])
    _same(cache, plain)
    K2, V2 = K[:, 30:33] * 0 + 448, V[:, 30:33] * 0 - 449   # the code's largest value, and just above
    cache.sp_cache_append(K2.cuda(), V2.cuda(), _i32(47))
    plain.append(K2, V2, [47])
    _same(cache, plain)


def _check_attention(sp, cache, Q, lens, max_len, scale=None, acc_in=None, **kw):
    """Output, lse and accumulated weights within what the roundings allow.

    A score is summed 16 products at a time: D / 16 + 4 roundings (factors included) of 2^-22 of the
    magnitudes' sum, d in all.  Scores off by d move a weight by 2 d of itself, so an output by
    4 d of the weighted magnitudes of the values (numerator and sum), and lse by d.  The weights
    are rounded once to binary16 for bf16 outputs, in two parts for f16 ones; what is below
    binary16's range is off by up to 2^-25 of the largest weight, for every token."""
    plain = ref.PlainCache(cache)
    D = Q.shape[-1]
    sc = D ** -0.5 if scale is None else scale
    want, want_lse, want_acc, mag, terms = (np.nan_to_num(x, nan=np.nan, posinf=np.inf, neginf=-np.inf) for x in plain.attention(
        Q, lens, max_len, sc, None if acc_in is None else acc_in.cpu().double().numpy()))
    B, n, Hq = Q.shape[:3]
    lse = torch.full((B, n, Hq), 7.0, device="cuda")
    acc = torch.full((B, cache.n_kv_heads, max_len), 7.0, device="cuda")
    vmax = np.nanmax(np.abs(np.nan_to_num(plain.v)) * 2.0 ** plain.ve.astype(float)[..., None, None])
    d = (D / 16 + 4) * 2.0 ** -22 * np.nan_to_num(terms) + 2.0 ** -21
    assert d.max() < 0.01                                  # or the bound says nothing
    p_round = 2.0 ** -11 if Q.dtype == torch.bfloat16 else 2.0 ** -21
    outs = []
    for with_acc in (True, False):
        O = cache.sp_cache_attention(Q.cuda(), _i32(*lens), max_len, scale, lse=lse,
                                     acc_in=acc_in if with_acc else None, acc_out=acc if with_acc else None, **kw)
        got = O.cpu().double().numpy()
        outs.append(got)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        err = np.abs(np.nan_to_num(got) - np.nan_to_num(want))
        allowed = (UNIT[Q.dtype] * np.abs(np.nan_to_num(want)) + (4 * d[..., None] + p_round) * np.nan_to_num(mag)
                   + max_len * 2.0 ** -25 * vmax + 2.0 ** -24)
        assert (err <= allowed).all(), (err / allowed).max()
        gl = lse.cpu().double().numpy()
        assert np.array_equal(np.isneginf(gl), np.isneginf(want_lse))
        fin = np.isfinite(want_lse)
        assert (np.abs(gl[fin] - want_lse[fin]) <= 2 * d[fin] + 2.0 ** -21 * np.abs(want_lse[fin])).all()
    ga = acc.cpu().double().numpy()
    assert np.array_equal(np.isnan(ga), np.isnan(want_acc))
    allowed = (4 * d.max((1, 2))[:, None, None] + 2.0 ** -21) * np.nan_to_num(want_acc) + 2.0 ** -100
    assert (np.abs(np.nan_to_num(ga) - np.nan_to_num(want_acc)) <= allowed).all()
    return outs[0]


def _filled(sp, lens, heads, dim, block, seed=0, dtype=torch.float16, spread=0.5):
    B, top = len(lens), max(max(lens), 1)
    cache = _cache(sp, B, top + block, heads, dim, block, seed)
    K, V = _kv(B, top, heads, dim, dtype, seed, spread)
    cache.sp_cache_append(K.cuda(), V.cuda(), torch.zeros(B, dtype=torch.int32, device="cuda"),
                          _i32(*lens))
    return cache


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,group,dim,block,n_q", [
    (1, 1, 64, 16, 1), (2, 4, 128, 32, 1), (3, 1, 128, 64, 1), (2, 8, 64, 32, 1), (1, 3, 128, 16, 3),
    (2, 5, 64, 64, 2), (1, 4, 128, 32, 7), (2, 1, 64, 16, 9), (1, 8, 128, 64, 8)])
def test_attention(sp, heads, group, dim, block, n_q, dtype):
    lens = [1, 2, 15, 16, 17, 64, 100, 333, 0]
    cache = _filled(sp, lens, heads, dim, block)
    g = torch.Generator().manual_seed(1)
    Q = torch.randn(len(lens), n_q, heads * group, dim, generator=g).to(dtype)
    acc_in = torch.rand(len(lens), heads, 400, generator=g).cuda()
    _check_attention(sp, cache, Q, lens, 400, acc_in=acc_in)


@pytest.mark.parametrize("n_q", [1, 4])
def test_attention_over_a_long_cache(sp, n_q):
    lens = [5000, 4097]
    cache = _filled(sp, lens, 2, 128, 32)
    Q = torch.randn(2, n_q, 4, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    _check_attention(sp, cache, Q, lens, 5000)


def test_attention_lengths_past_the_bounds(sp):
    lens = [100, 100, -5, 90]
    cache = _filled(sp, [100, 100, 100, 100], 1, 64, 16)
    Q = torch.randn(4, 2, 2, 64, generator=torch.Generator().manual_seed(1)).to(torch.float16)
    lens[1] = 10 ** 6                                      # past the table: what is there counts
    _check_attention(sp, cache, Q, lens, 96)


def test_attention_ignores_what_lies_past_the_end_and_in_absent_blocks(sp):
    lens = [50, 33, 64]
    cache = _filled(sp, [64, 64, 64], 2, 64, 16)
    cache.table[1, 1], cache.table[2, 0] = -1, 10 ** 5
    for b, n in enumerate(lens):                            # NaN in every place past the end
        for j in range(n, cache.table.shape[1] * 16):
            blk = int(cache.table[b, j // 16])
            if 0 <= blk < cache.k.shape[0]:
                cache.k[blk, :, j % 16] = 0x7f
                cache.v[blk, :, j % 16] = 0xff
    Q = torch.randn(3, 1, 2, 64, generator=torch.Generator().manual_seed(1)).to(torch.float16)
    out = _check_attention(sp, cache, Q, lens, 64)
    assert np.isfinite(out).all()


def test_attention_nan_of_the_calls_own_tokens_reaches_only_rows_that_see_it(sp):
    lens = [40, 16]
    cache = _filled(sp, lens, 1, 128, 16)
    for b, j, which in ((0, 38, "v"), (1, 14, "k"), (0, 39, "v")):
        getattr(cache, which)[int(cache.table[b, j // 16]), 0, j % 16, 5] = 0x7f
    Q = torch.randn(2, 4, 2, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    out = _check_attention(sp, cache, Q, lens, 40)
    assert np.isfinite(out[0, :2]).all() and np.isnan(out[0, 2:, :, 5]).all() and np.isnan(out[1, 2:]).all()


def test_attention_steep_scores_and_wide_scales(sp):
    # scores over hundreds of units in ascending order (the running maximum keeps rising), blocks
    # of values whose scales differ by powers of two up to 2^24
    B, L, D = 1, 300, 64
    cache = _cache(sp, B, L, 1, D, 16)
    K = torch.zeros(B, L, 1, D)
    K[0, :, 0, 0] = torch.linspace(-200, 200, L)
    V = torch.randn(B, L, 1, D, generator=torch.Generator().manual_seed(0))
    V *= torch.exp2((torch.arange(L) // 16 % 7 * 4 - 12).float())[None, :, None, None]
    cache.sp_cache_append(K.to(torch.bfloat16).cuda(), V.to(torch.bfloat16).cuda(), _i32(0))
    for slope in (1.0, -1.0, 0.01):
        Q = torch.zeros(B, 1, 1, D)
        Q[..., 0] = slope
        _check_attention(sp, cache, Q.to(torch.float16), [L], L, scale=1.0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_queries_of_any_size_and_stride(sp, dtype):
    lens = [77, 20]
    cache = _filled(sp, lens, 2, 64, 16)
    g = torch.Generator().manual_seed(1)
    big = torch.randn(2, 3, 4, 67, generator=g)
    big[0, 0] *= 1e-6
    Q = big.to(dtype)
    dev = Q.cuda()
    plain = _check_attention(sp, cache, Q[..., 3:], lens, 77)
    out = torch.full((2, 4, 3, 70), 9.0, dtype=dtype, device="cuda")
    view = out.transpose(1, 2)[..., 2:66]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    cache.sp_cache_attention(dev[..., 3:], _i32(*lens), 77, O=view, stream=stream)
    stream.synchronize()
    ref_out = cache.sp_cache_attention(dev[..., 3:].contiguous(), _i32(*lens), 77)
    assert torch.equal(view, ref_out)
    assert (out[..., :2] == 9).all() and (out[..., 66:] == 9).all()


def test_attention_accumulates_in_place_and_gives_the_same_bits_twice(sp):
    lens = [900, 300]
    cache = _filled(sp, lens, 2, 128, 32)
    Q = torch.randn(2, 1, 8, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    n = _i32(*lens)
    acc = torch.zeros(2, 2, 900, device="cuda")
    first = cache.sp_cache_attention(Q, n, 900, acc_in=acc, acc_out=acc).clone()
    once = acc.clone()
    assert torch.allclose(once.sum(-1), torch.full((2, 2), 4.0, device="cuda"), rtol=1e-5)   # 4 heads of weight 1
    out = cache.sp_cache_attention(Q, n, 900, acc_in=acc, acc_out=acc)
    assert torch.equal(out, first)
    want = 2 * once
    for b, length in enumerate(lens):                       # the call's own token starts from 0 again
        want[b, :, length - 1] = once[b, :, length - 1]
    assert torch.equal(acc, want)


@pytest.mark.parametrize("heads,dim,block", [(1, 64, 16), (2, 128, 32), (3, 64, 64), (2, 128, 64)])
@pytest.mark.parametrize("budget,recent", [(64, 16), (50, 0), (33, 33), (33, 100), (1, 0), (400, 8)])
def test_evict(sp, heads, dim, block, budget, recent):
    lens = [300, 64, 51, 1, 0, 299]
    cache = _filled(sp, lens, heads, dim, block)
    g = torch.Generator().manual_seed(budget)
    acc = torch.rand(len(lens), heads, 310, generator=g).pow(6)
    acc[0, 0, ::3] = acc[0, 0, 0]                           # ties across the cut
    acc[1, 0, 5:40] = 0.0
    acc[1, 0, 7] = -0.0
    acc[2, 0, 9], acc[2, 0, 11] = float("nan"), float("inf")
    _check_evict(sp, cache, lens, 310, acc, budget, recent)


def _check_evict(sp, cache, lens, max_len, acc, budget, recent):
    dst = _cache(sp, len(lens), budget, cache.n_kv_heads, cache.head_dim, cache.block_tokens, seed=9)
    plain, plain_dst = ref.PlainCache(cache), ref.PlainCache(dst)
    kept, acc_out, lens_out = cache.sp_cache_evict(_i32(*lens), max_len, acc.cuda(), budget, recent, dst)
    want = plain.evict(plain_dst, lens, max_len, acc.numpy(), budget, recent)
    assert np.array_equal(kept.cpu().numpy(), want)
    _same(dst, plain_dst)
    assert lens_out.tolist() == [max(0, min(n, budget, max_len)) for n in lens]
    moved = np.where(want >= 0, np.take_along_axis(acc.numpy(), np.maximum(want, 0), 2), 0.0)
    assert np.array_equal(acc_out.cpu().numpy(), moved, equal_nan=True)


@pytest.mark.parametrize("n,budget", [(5000, 600), (9000, 8999), (20000, 1), (16385, 4096)])
def test_evict_long_rows(sp, n, budget):
    cache = _filled(sp, [n, n - 77], 1, 64, 64)
    g = torch.Generator().manual_seed(n)
    acc = torch.randn(2, 1, n, generator=g)                 # any floats order
    acc[1] = torch.randint(0, 5, (1, n), generator=g).float()   # many ties
    _check_evict(sp, cache, [n, n - 77], n, acc, budget, min(32, budget))


def test_evict_equal_weights_keep_the_first(sp):
    cache = _filled(sp, [100], 1, 64, 16)
    kept, _, _ = cache.sp_cache_evict(_i32(100), 100, torch.ones(1, 1, 100, device="cuda"), 20, 4,
                                      sp.KvCache.empty(1, 20, 1, 64, 16))
    assert kept.flatten().tolist() == list(range(16)) + list(range(96, 100))


def test_attention_then_evict_then_attention(sp):
    # the tokens that receive all the attention survive, so the output hardly changes
    L, D = 256, 64
    cache = sp.KvCache.empty(1, L, 1, D, 16)
    K = torch.randn(1, L, 1, D, generator=torch.Generator().manual_seed(0))
    q = torch.randn(1, 1, 1, D, generator=torch.Generator().manual_seed(1))
    K[0, 10:20, 0] = q[0, 0] * 2
    V = torch.randn(1, L, 1, D, generator=torch.Generator().manual_seed(2))
    cache.sp_cache_append(K.to(torch.float16).cuda(), V.to(torch.float16).cuda(), _i32(0))
    Q = q.to(torch.float16).cuda()
    acc = torch.zeros(1, 1, L, device="cuda")
    before = cache.sp_cache_attention(Q, _i32(L), L, acc_in=acc, acc_out=acc)
    dst = sp.KvCache.empty(1, 64, 1, D, 16)
    kept, _, lens = cache.sp_cache_evict(_i32(L), L, acc, 32, 4, dst)
    assert set(range(10, 20)) <= set(kept.flatten().tolist())
    after = dst.sp_cache_attention(Q, lens, 32)
    gone = 1 - acc.flatten()[kept.flatten().long()].sum().item()
    assert (after - before).abs().max().item() <= 2 * gone * V.abs().max().item() + 0.02


def test_offsets_past_32_bits(sp):
    # pools of more than 2^32 bytes: the blocks in use are the last ones
    n, H, T, D = 34000, 16, 64, 128
    k = torch.empty(n, H, T, D, dtype=torch.uint8, device="cuda")
    v = torch.empty(n, H, T, D, dtype=torch.uint8, device="cuda")
    assert k.numel() > 2 ** 32
    ks, vs = (torch.ones(n, H, device="cuda") for _ in range(2))
    table = torch.tensor([[n - 1, 3, n - 2, 32767]], dtype=torch.int32, device="cuda")
    cache = sp.KvCache(k, v, ks, vs, table)
    K, V = _kv(1, 200, H, D, torch.bfloat16, 1, 0.3)
    cache.sp_cache_append(K.cuda(), V.cuda(), _i32(0))
    ids = table[0].long()
    small = sp.KvCache(k[ids].contiguous(), v[ids].contiguous(), ks[ids].contiguous(), vs[ids].contiguous(),
                       torch.arange(4, dtype=torch.int32, device="cuda").view(1, 4))
    other = sp.KvCache.empty(1, 256, H, D, T)
    other.sp_cache_append(K.cuda(), V.cuda(), _i32(0))
    assert torch.equal(small.k[:3], other.k[:3]) and torch.equal(small.v_scale, other.v_scale)
    Q = torch.randn(1, 1, 2 * H, D, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    assert torch.equal(cache.sp_cache_attention(Q, _i32(200), 200), other.sp_cache_attention(Q, _i32(200), 200))
    acc = torch.rand(1, H, 200, device="cuda")
    a, b = sp.KvCache.empty(1, 64, H, D, T), sp.KvCache.empty(1, 64, H, D, T)
    cache.sp_cache_evict(_i32(200), 200, acc, 50, 5, a)
    other.sp_cache_evict(_i32(200), 200, acc, 50, 5, b)
    assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v)


def test_binding_refusals(sp):
    cache = sp.KvCache.empty(2, 64, 2, 64, 16)
    x = torch.zeros(2, 1, 2, 64, dtype=torch.float16, device="cuda")
    n = _i32(5, 5)
    acc = torch.zeros(2, 2, 64, device="cuda")
    for bad in (lambda: cache.sp_cache_append(x.float(), x.float(), n), lambda: cache.sp_cache_append(x, x[:, :, :1], n),
                lambda: cache.sp_cache_append(x, x.to(torch.bfloat16), n), lambda: cache.sp_cache_append(x, x, n.long()),
                lambda: cache.sp_cache_append(x, x, _i32(1)), lambda: cache.sp_cache_append(x[:1], x[:1], n),
                lambda: cache.sp_cache_append(x.cpu(), x.cpu(), n),
                lambda: cache.sp_cache_attention(x[:, :, :1], n, 64), lambda: cache.sp_cache_attention(x[..., :32], n, 64),
                lambda: cache.sp_cache_attention(x, n, 64, scale=float("nan")),
                lambda: cache.sp_cache_attention(x, n, 65, acc_out=acc),
                lambda: cache.sp_cache_attention(x, n, 64, acc_out=acc, workspace=torch.zeros(8, device="cuda")),
                lambda: cache.sp_cache_attention(x, n, -1), lambda: cache.sp_cache_attention(x, n.cpu(), 64),
                lambda: cache.sp_cache_evict(n, 64, acc, 65, 0, cache.empty(2, 64, 2, 64, 16)),
                lambda: cache.sp_cache_evict(n, 64, acc, 32, 0, cache.empty(2, 64, 2, 128, 16)),
                lambda: cache.sp_cache_evict(n, 64, acc, 32, -1, cache.empty(2, 64, 2, 64, 16)),
                lambda: sp.KvCache(cache.k[..., :32].contiguous(), cache.v[..., :32].contiguous(), cache.k_scale,
                                   cache.v_scale, cache.table).sp_cache_append(x[..., :32], x[..., :32], n)):
        with pytest.raises(sp.SpError):
            bad()
