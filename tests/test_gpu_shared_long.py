"""Attention over shared prefixes where a block takes many steps of 64 tokens, against its definition in
binary64: rings that are used again and again, maxima and value scales that rise late."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = [torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def sp():
    from paper_2501_16376_b200 import binding
    binding.sp_wait_status(clear=True)
    yield binding
    assert binding.sp_wait_status() == 0                        # of everything in this file


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _cache(sp, n_seqs, cols, heads, dim, block, seed=0, spread=3, groups=None):
    """Random finite codes and scales over 2^-spread .. 2^spread; rows with blocks of their own, those
    of a group [(first, one past the last, blocks)] with the same first ones."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    table = torch.arange(n_seqs * cols).view(n_seqs, cols)
    for first, end, shared in groups or ():
        table[first:end, :shared] = table[first, :shared].clone()
    names, table = torch.unique(table, return_inverse=True)
    n = len(names) + 3
    order = torch.randperm(n, generator=torch.Generator().manual_seed(seed))
    shape = (n, heads, block, dim)
    k, v = ((torch.randn(shape, generator=g, device="cuda") * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            for _ in range(2))
    ks, vs = (torch.exp2(torch.randint(-spread, spread + 1, shape[:2], generator=g, device="cuda").float() - 7) for _ in range(2))
    return sp.KvCache(k, v, ks, vs, order[table].to(torch.int32).cuda())


def _queries(n_seqs, n_q, heads, dim, dtype, seed):
    return torch.randn(n_seqs, n_q, heads, dim, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def _exact(cache, Q, lens, max_len, scale):
    """(O, lse, weighted magnitudes of the values, largest sum of magnitudes behind a score), binary64;
    every row of the table as it stands."""
    B, n, Hq, D = Q.shape
    H, T = cache.n_kv_heads, cache.block_tokens
    O, mag = (torch.zeros(Q.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full(Q.shape[:3], float("-inf"), dtype=torch.float64, device="cuda")
    terms = torch.zeros_like(lse)
    for b in range(B):
        stored = max(0, min(int(lens[b]), max_len, cache.table.shape[1] * T))
        if stored == 0:
            continue
        ids = cache.table[b, :(stored + T - 1) // T].long()
        here = (ids >= 0) & (ids < cache.k.shape[0])
        ids = torch.where(here, ids, 0)
        dense = lambda c, s: (c[ids].view(torch.float8_e4m3fn).double() * s[ids].double()[..., None, None]).transpose(0, 1).reshape(H, -1, D)[:, :stored]
        K, V = dense(cache.k, cache.k_scale), dense(cache.v, cache.v_scale)
        q = Q[b].double().view(n, H, Hq // H, D).permute(1, 0, 2, 3)           # [H, n, group, D]
        S = torch.einsum("hngd,hjd->hngj", q, K) * scale
        size = torch.einsum("hngd,hjd->hngj", q.abs(), K.abs()) * abs(scale)
        at = torch.arange(stored, device="cuda")
        sees = (at <= int(lens[b]) - n + torch.arange(n, device="cuda")[:, None]) & here.repeat_interleave(T)[:stored]
        sees = sees[None, :, None]
        S = torch.where(sees, S, float("-inf"))
        top = S.amax(-1, keepdim=True)
        P = torch.where(sees, torch.exp(S - torch.where(top.isinf(), 0.0, top)), 0.0)
        total = P.sum(-1, keepdim=True)
        P = torch.where(total > 0, P / total, 0.0)
        back = lambda t: t.permute(1, 0, 2, 3).reshape(n, Hq, -1)
        O[b], mag[b] = back(torch.einsum("hngj,hjd->hngd", P, V)), back(torch.einsum("hngj,hjd->hngd", P, V.abs()))
        lse[b] = back(torch.where(total > 0, total.log() + top, float("-inf")))[..., 0]
        terms[b] = back(torch.where(sees, size, 0.0).amax(-1, keepdim=True))[..., 0]
    return O, lse, mag, terms


def _check(cache, Q, lens, max_len, starts, prefix, steps, scale=None, max_group=None):
    """Half a step of the output and, from there on, roundings.  A score is a sum of D products, 16 at a
    time, which the tensor cores cut to 2^-22: off by d = (D / 16 + 4) 2^-22 of its terms' magnitudes.  A
    weight is then off by 4 d of itself (weight and sum), by 2^-17 where it enters its product in two
    parts, by 2^-20 for the exponential and the additions.  An output is a sum of 8 products a step of 64
    tokens, each cut to 2^-22 of what it is added to.  steps: of a block, at most."""
    D = Q.shape[-1]
    sc = D ** -0.5 if scale is None else scale
    max_group = max(b - a for a, b in zip(starts, starts[1:])) if max_group is None else max_group
    lse = torch.full(Q.shape[:3], 77.0, device="cuda")
    O = cache.sp_cache_attention_shared(Q, _i32(lens), max_len, _i32(starts), _i32(prefix), max(prefix), max_group, scale=scale, lse=lse).double()
    want, want_lse, mag, terms = _exact(cache, Q, lens, max_len, sc)
    d = (D / 16 + 4) * 2.0 ** -22 * terms
    bound = torch.finfo(Q.dtype).eps / 2 * want.abs() + (4 * d[..., None] + 2.0 ** -17 + 2.0 ** -20 + 8 * steps * 2.0 ** -22) * mag
    bound += 2.0 ** (-25 if Q.dtype == torch.float16 else -134)
    # what the type cannot hold is infinite: its rounding from half a step past its largest value on
    largest = torch.finfo(Q.dtype).max * (1 + torch.finfo(Q.dtype).eps / 4)
    beyond, near = want.abs() - bound > largest, want.abs() + bound > largest
    assert torch.equal(O[beyond], want[beyond].sign() * float("inf")) and O[~near].isfinite().all()
    far = ((O - want).abs() > bound) & ~near
    assert not far.any(), (far.nonzero()[:4], O[far][:4], want[far][:4], bound[far][:4])
    empty = want_lse.isinf()
    assert torch.equal(lse.isinf(), empty)
    error = torch.where(empty, 0.0, lse.double() - torch.where(empty, 0.0, want_lse)).abs()
    assert (error <= d + 2.0 ** -20 * (1 + want_lse.abs())).all()
    return O


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size,dim", [(9, 64), (33, 128), (70, 64), (66, 128)])
def test_maximum_and_value_scale_rise_in_one_step(sp, size, dim, dtype):
    """40 (group, kv head) pairs each of two groups, so that a block takes all 16 steps of its prefix.  In the
    twelfth, the maximum rises by 2^16 in its first 32 tokens and by 2^16 again in its second 32, and in
    two of the runs the value scale by 2^45 as well (once past what binary16 holds): a rescaling that is lost
    leaves the earlier tokens' sums 2^16 times too large, with values that show it."""
    heads, block, group = 40, 32, 2
    shared = 32
    for early, later in ((4, -6), (-30, 15), (-44, 1)):
        starts = [0, size, size + 3]
        cache = _cache(sp, size + 3, shared + 1, heads, dim, block, seed=size, groups=[(0, size, shared), (size, size + 3, shared)])
        one = torch.ones(1).to(torch.float8_e4m3fn).view(torch.uint8).item()
        cache.k.zero_()
        cache.k_scale.fill_(1.0)
        cache.v_scale.fill_(2.0 ** early)
        for first in (0, size):
            row = cache.table[first].long()
            late = row[22:24]                                   # places 704 .. 767: the twelfth step
            cache.v_scale[late] = 2.0 ** later
            cache.k[late[0], :, 9, 0] = one                     # 16 above the rest
            cache.k[late[1], :, 20, :2] = one                   # 32 above
        Q = torch.zeros(size + 3, 1, heads * group, dim, device="cuda")
        Q[..., 0] = Q[..., 1] = 16.0
        lens = [shared * block + 1 + b % 20 for b in range(size + 3)]
        _check(cache, Q.to(dtype), lens, (shared + 1) * block, starts, [shared * block] * 2, 16, scale=0.6931471805599453)


@pytest.mark.parametrize("dtype", DTYPES)
def test_what_the_kernel_just_before_wrote(sp, dtype):
    """Many steps in one graph, each of which writes the queries, lengths, groups, tokens and counts that its
    attention reads, with nothing between them: all as with a wait before and after each kernel."""
    heads, dim, block, size, cols = 2, 64, 16, 24, 40
    steps = 12
    g = torch.Generator().manual_seed(3)
    cache = _cache(sp, size, cols, heads, dim, block, seed=5)
    cache = sp.KvCache(cache.k, cache.v, cache.k_scale, cache.v_scale, cache.table,
                       refs=torch.zeros(cache.k.shape[0], dtype=torch.int32, device="cuda"))
    cache.refs[cache.table.flatten().long()] = 1
    begin = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.table, cache.refs)]
    new = [torch.randn(size, 1, h, dim, generator=g).to(dtype).cuda() for h in (8, 2, 2)]
    freq = torch.ones(dim // 2, device="cuda")
    starts = [_i32([0, 6 + 3 * i, 20, size]) for i in range(2)]
    prefixes = [_i32([330 - 20 * i, 64, 200 + 40 * i]) for i in range(2)]
    lens0 = torch.randint(400, 600, (size,), generator=g, dtype=torch.int32).cuda()
    state = {}

    def reset():
        for t, b in zip((cache.k, cache.v, cache.k_scale, cache.v_scale, cache.table, cache.refs), begin):
            t.copy_(b)
        state.update(place=lens0.clone(), q=torch.empty_like(new[0]), k=torch.empty_like(new[1]),
                     start=starts[0].clone(), prefix=prefixes[0].clone())

    def run(wait):
        out, s, sync = [], state, (torch.cuda.synchronize if wait else lambda: None)
        for i in range(steps):
            s["start"].copy_(starts[i & 1])
            s["prefix"].copy_(prefixes[i & 1])
            cache.sp_cache_reserve(s["place"], 1)
            sync()
            sp.sp_qk_norm_rotary(new[0], new[1], s["place"], freq, Q_out=s["q"], K_out=s["k"])
            sync()
            cache.sp_cache_append(s["k"], new[2], s["place"])
            s["place"].add_(1)
            sync()
            out.append(cache.sp_cache_attention_shared(s["q"], s["place"], cols * block, s["start"], s["prefix"], 340, 20))
            sync()
        return out

    reset()
    want = [o.clone() for o in run(True)]
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(False)
    for _ in range(20):
        for t, b in zip((cache.k, cache.v, cache.k_scale, cache.v_scale, cache.table, cache.refs), begin):
            t.copy_(b)
        state["place"].copy_(lens0)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_the_same_from_call_to_call(sp):
    """Nothing in a call depends on which warp or block comes first."""
    for dtype, size, heads, group, dim in ((torch.bfloat16, 32, 8, 4, 128), (torch.float16, 40, 40, 1, 128), (torch.bfloat16, 70, 8, 4, 64)):
        cols, block = 66, 32
        cache = _cache(sp, 2 * size, cols, heads, dim, block, seed=size, groups=[(0, size, 62), (size, 2 * size, 60)])
        Q = _queries(2 * size, 1, heads * group, dim, dtype, size) * 2
        lens = _i32([62 * block + 1 + 5 * b % 70 for b in range(2 * size)])
        lse = torch.empty(Q.shape[:3], device="cuda")
        call = lambda: (cache.sp_cache_attention_shared(Q, lens, cols * block, _i32([0, size, 2 * size]), _i32([62 * block, 60 * block]),
                                                        62 * block, size, lse=lse), lse.clone())
        first = call()
        for _ in range(40):
            again = call()
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,group,n_q", [(2, 4, 1), (40, 1, 1), (2, 4, 4)])
@pytest.mark.parametrize("low,high", [(100, 500), (500, 100), (100, 655), (655, 100), (655, 640)])
def test_nan_far_below_the_maximum(sp, heads, group, n_q, low, high, dtype):
    """A NaN value whose weight lies 2^-200 below the largest, in another stretch of the prefix, in the
    tail, in the prefix under a maximum of the tail: it reaches its column of every row that sees it, as
    in sp_cache_attention."""
    size, block, shared = 5, 16, 40
    cache = _cache(sp, size, shared + 2, heads, 64, block, seed=7, groups=[(0, size, shared)])
    cache.k.zero_()
    cache.k_scale.fill_(1.0)
    one = torch.ones(1).to(torch.float8_e4m3fn).view(torch.uint8).item()
    for b in range(size):
        cache.k[cache.table[b, high // block].long(), :, high % block, 0] = one
        cache.v[cache.table[b, low // block].long(), :, low % block, 9] = 0x7f
    Q = torch.zeros(size, n_q, heads * group, 64, device="cuda")
    Q[..., 0] = 16.0
    lens = [672, 660, 657, 300, 660]
    scale = 200 / 16 * 0.6931471805599453
    call = dict(scale=scale)
    O = cache.sp_cache_attention_shared(Q.to(dtype), _i32(lens), 672, _i32([0, size]), _i32([shared * block]), shared * block, size, **call)
    alone = cache.sp_cache_attention(Q.to(dtype), _i32(lens), 672, **call)
    sees = torch.tensor([[x - n_q + i >= low for i in range(n_q)] for x in lens], device="cuda")
    want = torch.zeros(O.shape, dtype=torch.bool, device="cuda")
    want[..., 9] = sees[..., None]
    assert torch.equal(O.isnan(), want) and torch.equal(alone.isnan(), want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,size", [(2, 4), (40, 4), (40, 70)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan"), 2.0 ** 127])
def test_scales_that_no_row_sees(sp, bad, heads, size, dtype):
    """Blocks of the prefix behind the longest sequence hold whatever memory held: their scales count for
    nothing, as in sp_cache_attention, which does not read them."""
    block, shared = 16, 48
    cache = _cache(sp, size + 2, shared + 2, heads, 64, block, seed=8, groups=[(0, size, shared), (size, size + 2, shared)])
    for first in (0, size):
        row = cache.table[first].long()
        cache.k_scale[row[33:]] = bad
        cache.v_scale[row[33:]] = bad
    lens = [33 * block - b % 9 for b in range(size + 1)] + [7]
    _check(cache, _queries(size + 2, 1, heads, 64, dtype, 8), lens, (shared + 2) * block, [0, size, size + 2], [shared * block] * 2, 12)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [2, 16, 32])
def test_sums_of_long_prefixes_do_not_shrink(sp, size, dtype):
    """75 groups (so that the device has a block for every one) of one prefix of 131072 tokens, positive
    values.  The tensor cores cut what they add to: at most 1024 products (128 steps) in a row take less
    than 2^-13 off (each less than 2^-23), and 2^-15 on average (a cut is half of that, a sum half of its
    last value).  With scores of deviation 2.4 some 400 tokens count, outputs of a column differ from row to
    row by more than the type's steps, and their own roundings have a mean of 0 (six deviations of it
    are allowed); with an eighth of that they nearly agree and round alike, so their mean says nothing."""
    groups, heads, T, tokens = 75, 8, 64, 131072
    g = torch.Generator(device="cuda").manual_seed(size)
    shape = (tokens // T, 1, T, 64)
    k = (torch.randn(shape, generator=g, device="cuda") * 40).to(torch.float8_e4m3fn)
    v = (torch.rand(shape, generator=g, device="cuda") * 200 + 100).to(torch.float8_e4m3fn)
    one = torch.full(shape[:2], 2.0 ** -7, device="cuda")
    table = torch.arange(shape[0], dtype=torch.int32, device="cuda").repeat(groups * size, 1)
    cache = sp.KvCache(k.view(torch.uint8), v.view(torch.uint8), one, one.clone(), table)
    Q = _queries(groups * size, 1, heads, 64, dtype, size)
    K, V = (x.view(-1, 64).double() * 2.0 ** -7 for x in (k, v))
    rows = torch.randperm(groups * size * heads, generator=torch.Generator().manual_seed(1))[:1024].cuda()
    for scale in (1 / 8, 1.0):
        O = cache.sp_cache_attention_shared(Q, _i32([tokens] * (groups * size)), tokens, _i32([i * size for i in range(groups + 1)]),
                                            _i32([tokens] * groups), tokens, size, scale=scale)
        want = torch.softmax(Q.view(-1, 64)[rows].double() @ K.T * scale, -1) @ V
        error = (O.view(-1, 64)[rows].double() - want) / want
        assert error.abs().max() <= torch.finfo(dtype).eps / 2 + 2.0 ** -13
    assert error.mean().abs() <= 2.0 ** -15 + 6 * torch.finfo(dtype).eps / 2 / error.numel() ** 0.5


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("size", [10, 25, 50])
def test_blocks_of_many_steps(sp, size, dim, dtype):
    """8 groups of 16 kv heads, a block for each with all 24 steps of its prefix: 40, 100 and 200 rows.  Random
    scores; scores that rise with every step, by less and by more than a weight may exceed the maximum;
    value scales that rise by 2^45 in the 17th step."""
    heads, block, group, groups, shared = 16, 32, 4, 8, 47
    n, tokens = groups * size, 47 * 32
    starts = [i * size for i in range(groups + 1)]
    cache = _cache(sp, n, shared + 2, heads, dim, block, seed=size, groups=[(a, a + size, shared) for a in starts[:-1]])
    Q = _queries(n, 1, heads * group, dim, dtype, size)
    lens = [tokens + 1 + (7 * b) % 64 if b % 9 else 700 + 11 * (b % 50) for b in range(n)]
    call = dict(lens=lens, max_len=tokens + 64, starts=starts, prefix=[tokens + 5 * (i % 3) for i in range(groups)], steps=24)
    _check(cache, Q, **call)
    begin = cache.v_scale.clone()
    for first in starts[:-1]:
        cache.v_scale[cache.table[first, 34:].long()] *= 2.0 ** 45
    if dtype == torch.float16:
        cache.v_scale *= 2.0 ** -45
    _check(cache, Q, **call)
    cache.v_scale.copy_(begin)
    place = torch.arange(tokens + 64).view(-1, block)
    codes = torch.stack([place // 128, place // 64 % 2, place % 64 // 8], -1).float().to(torch.float8_e4m3fn).view(torch.uint8).cuda()
    for b in range(n):
        cache.k[cache.table[b].long(), :, :, :3] = codes[:, None]
    scale = cache.k_scale.fill_(1.0)
    cache.k[..., 3:] = 0
    for rise in (4.0, 24.0):
        Q[..., 0], Q[..., 1], Q[..., 2] = 2 * rise, rise, rise / 8
        _check(cache, Q, scale=1.0, **call)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n_q,max_group", [(1, 9), (2, 9), (1, 3)])
def test_a_hundred_groups_of_all_sizes(sp, n_q, max_group, dtype):
    """Groups of 0 to 9 sequences, prefixes from nothing to all of a sequence, sequences of no group before and
    behind them, sequences past max_group."""
    g = torch.Generator().manual_seed(n_q)
    sizes = [int(x) for x in torch.randint(0, 10, (100,), generator=g)]
    starts = [3]
    for s in sizes:
        starts.append(starts[-1] + s)
    n, block, cols = starts[-1] + 5, 16, 30
    prefix = [int(x) for x in torch.randint(0, 29 * block, (100,), generator=g)]
    cache = _cache(sp, n, cols, 3, 64, block, seed=n_q, groups=[(a, b, p // block) for a, b, p in zip(starts, starts[1:], prefix) if b > a])
    lens = [int(x) for x in torch.randint(0, cols * block + 1, (n,), generator=g)]
    _check(cache, _queries(n, n_q, 6, 64, dtype, 1), lens, cols * block, starts, prefix, 8, max_group=max_group)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,group,dim", [(2, 4, 128), (40, 1, 64), (8, 12, 64)])
def test_long_tails_beside_a_long_prefix(sp, heads, group, dim, dtype):
    """A sequence of no group and a group with a short prefix beside a group with a long one: their tails are
    nearly all they have, many steps for one warp.  bf16 queries with channels far below the largest too."""
    block, cols, size = 64, 126, 12
    starts, prefix = [0, size, size + 3], [8000, 64]
    cache = _cache(sp, size + 4, cols, heads, dim, block, seed=heads, groups=[(0, size, 125), (size, size + 3, 1)])
    lens = [8001 + 3 * b for b in range(size)] + [3000, 3217, 64, 8000]
    Q = _queries(size + 4, 1, heads * group, dim, dtype, heads)
    _check(cache, Q, lens, cols * block, starts, prefix, 125)
    if dtype == torch.bfloat16:
        cache.k[..., 5] = 0
        Q[::2, ..., 5] = 2.0 ** 100
        Q[1::3, ..., :3] *= 2.0 ** -60
        _check(cache, Q, lens, cols * block, starts, prefix, 125)


@pytest.mark.parametrize("size", [6, 40, 70])
def test_value_scales_that_others_see(sp, size):
    """bf16: sequences that end before blocks whose value scales lie 2^100 above theirs."""
    heads, block, shared = 40, 32, 36
    cache = _cache(sp, size + 2, shared + 1, heads, 64, block, seed=size, groups=[(0, size, shared), (size, size + 2, shared)])
    for first in (0, size):
        row = cache.table[first].long()
        cache.v_scale[row[:20]] *= 2.0 ** -60
        cache.v_scale[row[20:]] = 2.0 ** 37
        cache.v_scale[row[:20]] = cache.v_scale[row[:20]].clamp(min=2.0 ** -63)
    lens = [(20 * block - b % 40) if b % 3 else (shared * block + 1 + b % 20) for b in range(size + 2)]
    _check(cache, _queries(size + 2, 1, heads * 2, 64, torch.bfloat16, size), lens, (shared + 1) * block, [0, size, size + 2],
           [shared * block] * 2, 18)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n_q,group", [(2, 4), (4, 4), (5, 4), (40, 4)])
def test_sequences_alone_of_few_and_many_queries(sp, n_q, group, dtype):
    """Groups of one on both sides of the rule for them: 8, 16, 20 and 160 rows, 16 and 40 (sequence, kv head)."""
    for heads, size in ((8, 2), (8, 5)):
        cache = _cache(sp, size, 40, heads, 64, 32, seed=n_q)
        lens = [1280 - 7 * b for b in range(size)]
        _check(cache, _queries(size, n_q, heads * group, 64, dtype, n_q), lens, 1280, list(range(size + 1)), [1200 - 40 * b for b in range(size)], 19)
