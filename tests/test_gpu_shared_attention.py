"""Attention over shared prefixes against its definition in binary64."""
import numpy as np
import pytest
import torch

from . import answers_reference as answers
from . import serve_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = [torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def sp():
    from paper_2501_16376_b200 import binding
    return binding


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _cache(sp, n_seqs, cols, heads, dim, block, seed=0, spread=4):
    """Random finite codes, scales over 2^-spread .. 2^spread, every row with blocks of its own."""
    g = torch.Generator().manual_seed(seed)
    n = n_seqs * cols + 3
    shape = (n, heads, block, dim)
    k, v = ((torch.randn(shape, generator=g) * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).cuda() for _ in range(2))
    ks, vs = (torch.exp2(torch.randint(-spread, spread + 1, shape[:2], generator=g).float() - 7).cuda() for _ in range(2))
    table = torch.randperm(n, generator=g)[:n_seqs * cols].view(n_seqs, cols).to(torch.int32).cuda()
    return sp.KvCache(k, v, ks, vs, table)


def _queries(n_seqs, n_q, heads, dim, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(n_seqs, n_q, heads, dim, generator=g).to(dtype)


def _check(sp, cache, Q, lens, max_len, starts, prefix, max_prefix=None, max_group=None, scale=None, stream=None, **kw):
    """Half a step of the output and, from there on, roundings of 2^-24.  A score is a sum of D products
    (16 at a time, tensor cores cutting what they add to 2^-22: D / 16 + 4 steps): off by
    d = (D / 16 + 4) 2^-22 of its terms' magnitudes.  A weight is then off by 2 d of itself (weight and
    sum), by 2^-17 where it enters its product in two parts of 8 bits, and by 2^-20 for the exponential
    and the additions (up to 2^4 of 2^-24 a tile, few tiles); lse by d and 2^-20 of 1 + |lse|."""
    max_prefix = max(list(prefix) + [0]) if max_prefix is None else max_prefix
    max_group = max([b - a for a, b in zip(starts, starts[1:])] + [0]) if max_group is None else max_group
    plain = ref.PlainCache(cache)
    plain.table = answers.shared_table(plain.table, plain.T, starts, prefix, max_prefix, max_group)
    D = Q.shape[-1]
    sc = D ** -0.5 if scale is None else scale
    want, want_lse, _, mag, terms = plain.attention(Q, lens, max_len, sc)
    lse = torch.full(Q.shape[:3], 77.0, device="cuda")
    O = cache.sp_cache_attention_shared(Q.cuda(), _i32(lens), max_len, _i32(list(starts)), _i32(list(prefix)), max_prefix, max_group,
                                        scale=scale, lse=lse, **kw)
    O, lse = O.double().cpu().numpy(), lse.double().cpu().numpy()
    d = (D / 16 + 4) * 2.0 ** -22 * terms
    bound = torch.finfo(Q.dtype).eps / 2 * np.abs(want) + (2 * d[..., None] * 2 + 2.0 ** -17 + 2.0 ** -20) * mag
    bound += 2.0 ** (-25 if Q.dtype == torch.float16 else -134)             # half the type's least step
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(O), nan)
    far = np.abs(O - want) > bound
    assert not far[~nan].any(), (np.argwhere(far & ~nan)[:4], O[far & ~nan][:4], want[far & ~nan][:4], bound[far & ~nan][:4])
    empty = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(lse), empty) and not O[empty].any()
    ok = ~empty & ~np.isnan(want_lse)
    assert (np.abs(lse - want_lse)[ok] <= (d + 2.0 ** -20 * (1 + np.abs(np.where(empty, 0, want_lse))))[ok]).all()
    return O


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,group,dim,block", [(1, 1, 64, 16), (2, 4, 128, 32), (3, 5, 64, 32), (1, 8, 128, 64), (2, 1, 128, 16)])
@pytest.mark.parametrize("n_q", [1, 3])
def test_groups_of_all_kinds(sp, heads, group, dim, block, n_q, dtype):
    """Groups of 1, 5 and no sequences, prefixes that end inside a block, two sequences of no group."""
    starts, prefix = [0, 1, 6, 6], [3 * block + 7, 5 * block, block]
    lens = [3 * block + 9, 5 * block + 1, 6 * block, 5 * block + 30, 5 * block + n_q, 7 * block - 1, 45, 2 * block]
    cache = _cache(sp, 8, 8, heads, dim, block, seed=dim + block)
    Q = _queries(8, n_q, heads * group, dim, dtype, n_q)
    _check(sp, cache, Q, lens, max(lens), starts, prefix)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size,group,n_q,dim", [(3, 1, 1, 64), (17, 1, 1, 128), (33, 2, 1, 64), (40, 4, 1, 128), (23, 3, 2, 64), (70, 4, 1, 64), (65, 4, 2, 128)])
def test_rows_of_a_group(sp, size, group, n_q, dim, dtype):
    """3 to 520 query rows for one prefix of an odd number of blocks."""
    cache = _cache(sp, size + 1, 15, 1, dim, 16, seed=size)
    prefix = 13 * 16
    lens = [prefix + 1 + (7 * b) % 29 for b in range(size)] + [100]
    Q = _queries(size + 1, n_q, group, dim, dtype, size)
    _check(sp, cache, Q, lens, 240, [0, size], [prefix])


@pytest.mark.parametrize("dtype", DTYPES)
def test_long_prefixes(sp, dtype):
    cache = _cache(sp, 4, 130, 2, 64, 64, seed=1)
    lens = [8001, 8320, 8192, 7777]
    Q = _queries(4, 1, 4, 64, dtype, 5)
    _check(sp, cache, Q, lens, 8320, [0, 3, 4], [8000, 7000])


def test_sequences_that_end_inside_the_prefix(sp):
    """Queries see the tokens up to their own place only, whatever lies behind: NaN, infinite scales."""
    block = 16
    for dtype in DTYPES:
        cache = _cache(sp, 6, 12, 2, 64, block, seed=2)
        rows = cache.table[0].long()
        cache.k[rows[6], :, 3:], cache.v[rows[6], :, 3:] = 0x7f, 0xff       # from place 99 on
        cache.v[rows[7:9]] = 0x7f
        lens = [99, 0, 50, 97, -4, 2]
        for n_q in (1, 4):
            Q = _queries(6, n_q, 4, 64, dtype, 3)
            O = _check(sp, cache, Q, lens, 192, [0, 6], [160])
            assert np.isfinite(O).all()


def test_nan_in_the_prefix_reaches_those_who_see_it(sp):
    for dtype in DTYPES:
        cache = _cache(sp, 3, 10, 1, 64, 16, seed=3)
        row = cache.table[0].long()
        cache.v[row[5], 0, 2, 9] = 0x7f                                     # value of place 82, column 9
        Q = _queries(3, 2, 2, 64, dtype, 4)
        O = _check(sp, cache, Q, [83, 84, 150], 160, [0, 3], [144])
        assert np.isnan(O[1:, :, :, 9]).all() and np.isfinite(O[0, 0]).all() and np.isnan(O[0, 1, :, 9]).all()
        assert np.isfinite(np.delete(O, 9, -1)).all()
        cache.k[row[1], 0, 4, 0] = 0x7f                                     # a key of place 20: every row
        O = _check(sp, cache, Q, [83, 84, 150], 160, [0, 3], [144])
        assert np.isnan(O).all()


def test_blocks_that_the_table_does_not_name(sp):
    for block in (16, 32, 64):
        cache = _cache(sp, 4, 9, 2, 128, block, seed=4)
        cache.table[0, 1], cache.table[0, 4], cache.table[2, 7], cache.table[3, 0] = -1, 10 ** 6, -3, -1
        Q = _queries(4, 1, 4, 128, torch.bfloat16, 5)
        _check(sp, cache, Q, [8 * block, 6 * block + 1, 9 * block, 5], 9 * block, [0, 3], [6 * block])
        cache.table[0, :6] = -1
        _check(sp, cache, Q, [8 * block, 6 * block + 1, 9 * block, 6 * block], 9 * block, [0, 4], [6 * block])


def test_bounds_smaller_than_the_groups(sp):
    """Sequences past max_group and tokens past max_prefix are read through the sequences' own rows."""
    cache = _cache(sp, 9, 8, 2, 64, 16, seed=6)
    Q, lens = _queries(9, 1, 4, 64, torch.float16, 6), [100, 120, 128, 97, 100, 101, 128, 99, 5]
    for max_prefix, max_group in ((96, 3), (50, 8), (0, 8), (96, 0), (15, 2)):
        _check(sp, cache, Q, lens, 128, [0, 6, 9], [96, 64], max_prefix, max_group)
    _check(sp, cache, Q, lens, 110, [0, 6, 9], [96, 64])                    # max_len below some lengths
    _check(sp, cache, Q, lens, 128, [0, 6, 9], [1000, -5], 1000)            # past the table; negative
    _check(sp, cache, Q, lens, 128, [0], [], 100, 4)                        # no groups at all


def test_large_scores_and_scales_far_apart(sp):
    """Scores in the hundreds that rise along the prefix; value scales 2^60 apart, blocks of zeros."""
    for dtype in DTYPES:
        cache = _cache(sp, 5, 14, 1, 64, 16, seed=7)
        for i in range(12):
            cache.k_scale[cache.table[0, i].long()] *= 2.0 ** (i // 2)
        Q = _queries(5, 1, 6, 64, dtype, 7)
        lens = [200, 193, 224, 210, 100]
        _check(sp, cache, Q, lens, 224, [0, 5], [192], scale=0.5)
        cache = _cache(sp, 5, 14, 1, 64, 16, seed=8)
        row = cache.table[0].long()
        cache.v_scale[row[2]], cache.v_scale[row[3]], cache.v_scale[row[7]] = 2.0 ** -100, 2.0 ** -20, 2.0 ** 20
        cache.v[row[5]], cache.v_scale[row[5]] = 0, 2.0 ** -126
        _check(sp, cache, Q if dtype == torch.bfloat16 else Q, lens, 224, [0, 5], [112])
        if dtype == torch.bfloat16:
            cache.v_scale.copy_(torch.full_like(cache.v_scale, 2.0 ** -110))   # all far below 1
            _check(sp, cache, Q, lens, 224, [0, 5], [192])


def test_values_that_cancel(sp):
    """Two tokens share the attention and their values cancel; what is left is made of small weights."""
    for dtype in DTYPES:
        cache = _cache(sp, 2, 6, 1, 64, 16, seed=9, spread=0)
        row = cache.table[0].long()
        cache.k[row[0], 0, 1] = cache.k[row[0], 0, 0]
        cache.v[row[0], 0, 1] = cache.v[row[0], 0, 0] ^ 0x80
        Q = (cache.k[row[0], 0, 0].view(torch.float8_e4m3fn).float() / 16).to(dtype).cpu().view(1, 1, 1, 64).repeat(2, 1, 4, 1)
        _check(sp, cache, Q, [90, 96], 96, [0, 2], [80])


def test_small_channels_of_queries(sp):
    """bf16 channels far below the row's largest count where the keys are 0 in the large ones."""
    cache = _cache(sp, 3, 6, 1, 64, 16, seed=10, spread=0)
    cache.k[:, :, :, 0] = 0
    Q = _queries(3, 1, 2, 64, torch.bfloat16, 11)
    Q[..., 0] = 2.0 ** 100
    _check(sp, cache, Q, [90, 96, 81], 96, [0, 3], [80])


def test_one_token_and_none(sp):
    for block in (16, 64):
        cache = _cache(sp, 3, 2, 1, 128, block, seed=12)
        Q = _queries(3, 1, 2, 128, torch.bfloat16, 12)
        _check(sp, cache, Q, [1, 1, 1], 1, [0, 3], [block])
        _check(sp, cache, Q, [1, 0, block], 2 * block, [0, 3], [block])
        _check(sp, cache, Q, [block, block + 1, 2 * block], 2 * block, [0, 3], [1])
        _check(sp, cache, Q, [block, 5, 7], 0, [0, 3], [block])
    assert cache.sp_cache_attention_shared(Q[:, :0].cuda(), _i32([1, 1, 1]), 4, _i32([0, 3]), _i32([64]), 64, 3).shape == (3, 0, 2, 128)


def test_strided_queries_and_outputs(sp):
    cache = _cache(sp, 4, 8, 2, 64, 16, seed=13)
    g = torch.Generator().manual_seed(13)
    fused = torch.randn(4, 2, 10, 65, generator=g).to(torch.bfloat16)
    Q = fused[:, :, 2:8, 1:]
    out = torch.full((6, 4, 2, 66), 7.0, dtype=torch.bfloat16, device="cuda")
    O = out.permute(1, 2, 0, 3)[..., 1:65]
    dev = fused.cuda()
    plain = _check(sp, cache, Q, [100, 128, 97, 110], 128, [0, 4], [96])
    cache.sp_cache_attention_shared(dev[:, :, 2:8, 1:], _i32([100, 128, 97, 110]), 128, _i32([0, 4]), _i32([96]), 96, 4, O=O)
    assert np.array_equal(O.double().cpu().numpy(), plain)
    assert (out[..., 0] == 7).all() and (out[..., 65] == 7).all()


def test_the_same_as_attention_of_each_alone(sp):
    """On tables that do share their blocks, sp_cache_attention gives the same up to a rounding."""
    cache = _cache(sp, 6, 20, 4, 128, 32, seed=14)
    cache.table[1:, :15] = cache.table[:1, :15]
    Q, lens = _queries(6, 1, 16, 128, torch.float16, 14).cuda(), _i32([500, 640, 481, 600, 555, 490])
    a = cache.sp_cache_attention(Q, lens, 640).float()
    b = cache.sp_cache_attention_shared(Q, lens, 640, _i32([0, 6]), _i32([490]), 490, 6).float()
    assert (a - b).norm() <= 2.0 ** -11 * a.norm()


def test_captured_replays_and_streams(sp):
    cache = _cache(sp, 5, 12, 2, 64, 16, seed=15)
    Q, lens, starts, prefix = _queries(5, 1, 4, 64, torch.bfloat16, 15).cuda(), _i32([150, 160, 170, 180, 190]), _i32([0, 5]), _i32([144])
    call = lambda **kw: cache.sp_cache_attention_shared(Q, lens, 192, starts, prefix, 160, 5, **kw)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O = call()
        O2 = call()
    for add in (0, 1, 1):
        lens.add_(add)
        graph.replay()
        want = call()
        assert torch.equal(O, want) and torch.equal(O2, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    there = call(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(there, want)


def test_waits_have_not_run_out(sp):
    assert sp.sp_wait_status() == 0


@pytest.mark.parametrize("log2", [10, 23, 25, 27, 29, 31, 40, 60])
def test_one_token_far_above_the_others(sp, log2):
    """Scores of 2^log2 at one or two tokens and 0, or small ones, at the others: the output is their
    values' mean whatever the maximum's own rounding comes to."""
    for dtype in DTYPES:
        cache = _cache(sp, 3, 14, 1, 64, 16, seed=20, spread=0)
        row = cache.table[0].long()
        one = torch.tensor(1.0).to(torch.float8_e4m3fn).view(torch.uint8).item()
        cache.k[:] = 0
        cache.k_scale[:] = 1.0
        cache.k[row[3], 0, 5, 0] = cache.k[row[9], 0, 1, 0] = one
        cache.k[row[4], 0, 2, 0] = one | 0x80                              # as far below
        cache.k[:, :, :, 1] = one                                          # a term that all have
        Q = torch.zeros(3, 1, 4, 64)
        Q[..., 0], Q[..., 1] = 1.5, 0.25
        O = cache.sp_cache_attention_shared(Q.to(dtype).cuda(), _i32([224, 200, 193]), 224, _i32([0, 3]), _i32([192]), 192, 3,
                                            scale=2.0 ** log2).double().cpu()
        v = cache.v.view(torch.float8_e4m3fn).double() * cache.v_scale.double()[..., None, None]
        want = ((v[row[3], 0, 5] + v[row[9], 0, 1]) / 2).cpu()
        assert ((O - want).abs() <= torch.finfo(dtype).eps / 2 * want.abs() + 2.0 ** -17 * v.abs().max().cpu()).all()
        far = cache.sp_cache_attention_shared(-Q.to(dtype).cuda(), _i32([224, 200, 193]), 224, _i32([0, 3]), _i32([192]), 192, 3,
                                              scale=-2.0 ** log2).double().cpu()
        assert torch.equal(far, O)                                         # a negative scale


def test_scores_that_rise_by_a_little_and_by_much(sp):
    """The maximum is raised within a step and between steps, by less and by more than a weight may exceed it."""
    for dtype in DTYPES:
        for rise in (0.05, 0.3, 1.0, 4.0):
            cache = _cache(sp, 2, 20, 1, 64, 16, seed=21, spread=0)
            cache.k[:] = 0
            cache.k_scale[:] = 2.0 ** -4
            place = torch.arange(320).view(20, 16)
            row = cache.table[0].long().cpu()
            codes = (place.float() * rise).clamp(max=448).to(torch.float8_e4m3fn).view(torch.uint8)
            for i in range(20):
                cache.k[row[i], 0, :, 3] = codes[i].cuda()
            Q = torch.zeros(2, 1, 3, 64)
            Q[..., 3] = 8.0
            _check(sp, cache, Q.to(dtype), [320, 311], 320, [0, 2], [304], scale=1.0)


def test_more_rows_than_a_block_takes(sp):
    """2400 query rows of one prefix, the sequences of a group past 256 rows and 128."""
    cache = _cache(sp, 300, 6, 1, 64, 16, seed=22)
    lens = [64 + 1 + (5 * b) % 32 for b in range(300)]
    _check(sp, cache, _queries(300, 1, 8, 64, torch.bfloat16, 22), lens, 96, [0, 300], [64])


def test_pools_and_batches_of_nothing(sp):
    cache = sp.KvCache.pool(3, 64, 0, 2, 64, 16)
    Q = _queries(3, 1, 4, 64, torch.float16, 23).cuda()
    lse = torch.zeros(3, 1, 4, device="cuda")
    O = cache.sp_cache_attention_shared(Q, _i32([5, 64, 0]), 64, _i32([0, 3]), _i32([48]), 48, 3, lse=lse)
    assert not O.any() and torch.isneginf(lse).all()
    cache = sp.KvCache.pool(0, 64, 4, 2, 64, 16)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert cache.sp_cache_attention_shared(Q[:0], none, 64, _i32([0]), none, 48, 3).shape == (0, 1, 4, 64)
    cache.sp_cache_fork(none)
    assert cache.sp_cache_reserve(none, 5).tolist() == [0, 4] and cache.sp_cache_compact().item() == 0


def test_calls_on_two_streams_at_once(sp):
    """Two caches of other sizes and types on two streams, each as it is alone, again and again."""
    jobs = []
    for seed, (heads, dim, block, dtype, size) in enumerate(((2, 64, 16, torch.float16, 20), (4, 128, 32, torch.bfloat16, 40))):
        cache = _cache(sp, size, 20, heads, dim, block, seed=30 + seed)
        Q = _queries(size, 1, heads * 4, dim, dtype, seed).cuda()
        n = 16 * block
        lens = _i32([n + 1 + b % (3 * block) for b in range(size)])
        call = lambda cache=cache, Q=Q, lens=lens, n=n, size=size, block=block: cache.sp_cache_attention_shared(
            Q, lens, 20 * block, _i32([0, size]), _i32([n]), n, size)
        jobs.append((call, call()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    outs = [[], []]
    for _ in range(30):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                outs[i].append(jobs[i][0]())
    torch.cuda.synchronize()
    for (_, want), got in zip(jobs, outs):
        assert all(torch.equal(want, o) for o in got)


def test_buffers_that_change_between_calls(sp):
    """Queries, lengths, groups, table and scales of other values in the same memory from call to call,
    with nothing waited for between them: each call as it is with its own alone."""
    size, heads, dim, block, cols = 40, 2, 64, 16, 24
    base = _cache(sp, size, cols, heads, dim, block, seed=40)
    freq = torch.ones(dim // 2, device="cuda")
    cases = []
    for i in range(3):
        g = torch.Generator().manual_seed(50 + i)
        cases.append(dict(
            q=torch.randn(size, 1, heads * 4, dim, generator=g).half().cuda(), k=torch.randn(size, 1, heads, dim, generator=g).half().cuda(),
            table=torch.randperm(base.k.shape[0], generator=g)[:size * cols].view(size, cols).to(torch.int32).cuda(),
            place=torch.randint(200, cols * block - 1, (size,), generator=g, dtype=torch.int32).cuda(),
            starts=_i32([0, 10 + 5 * i, 40]), prefix=_i32([192 - 32 * i, 160 + 16 * i])))
    def run(into, of, wait):
        for name in into:
            into[name].copy_(of[name])
        for name, t in (("k", cache.k), ("v", cache.v), ("k_scale", cache.k_scale), ("v_scale", cache.v_scale)):
            t.copy_(getattr(base, name))
        cache.table.copy_(into["table"])
        if wait:
            torch.cuda.synchronize()
        lens = into["place"] + 1
        sp.sp_qk_norm_rotary(into["q"], into["k"], into["place"], freq, Q_out=into["q"], K_out=into["k"])
        cache.sp_cache_append(into["k"], into["k"], into["place"])
        if wait:
            torch.cuda.synchronize()
        return cache.sp_cache_attention_shared(into["q"], lens, cols * block, into["starts"], into["prefix"], 192, 30)
    cache = sp.KvCache(base.k.clone(), base.v.clone(), base.k_scale.clone(), base.v_scale.clone(), base.table.clone())
    into = {name: t.clone() for name, t in cases[0].items()}
    want = [run({name: t.clone() for name, t in c.items()}, c, True) for c in cases]
    got = [(i % 3, run(into, cases[i % 3], False)) for i in range(60)]
    for i, o in got:
        assert torch.equal(o, want[i])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size,prefix,tail,heads,group,n_q", [(1, 9000, 300, 1, 5, 3), (2, 4500, 10, 1, 1, 1), (2, 9000, 300, 1, 5, 3), (2, 40, 2000, 2, 2, 1), (8, 3000, 200, 2, 8, 4), (1, 40, 2000, 2, 2, 1)])
def test_few_rows_of_many_parts(sp, dtype, size, prefix, tail, heads, group, n_q):
    cols = -(-(prefix + tail) // 64)
    cache = _cache(sp, size, cols, heads, 64, 64, seed=size)
    lens = [prefix + tail - 7 * b for b in range(size)]
    _check(sp, cache, _queries(size, n_q, heads * group, 64, dtype, size), lens, cols * 64, [0, size], [prefix])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,group,n_q", [(4, 2, 1), (3, 8, 1), (2, 3, 4)])
def test_groups_of_one(sp, dtype, heads, group, n_q):
    """Every sequence alone: with enough kv heads and few rows, and otherwise."""
    cache = _cache(sp, 4, 40, heads, 64, 32, seed=60 + heads)
    _check(sp, cache, _queries(4, n_q, heads * group, 64, dtype, heads), [1280, 1100, 5, 700], 1280, [0, 1, 2, 3, 4], [1000, 1090, 64, 33])
