"""Shared blocks of the 8-bit cache (fork, reserve, compact) against a walk in Python."""
import random

import pytest
import torch

from . import answers_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2501_16376_b200 import binding
    return binding


def _pool(sp, n_seqs, cols, n_blocks, heads=2, dim=64, block=16, seed=0):
    """A pool of stale bytes with an empty table."""
    cache = sp.KvCache.pool(n_seqs, cols * block, n_blocks, heads, dim, block)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for t in (cache.k, cache.v):
        t.copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    for t in (cache.k_scale, cache.v_scale):
        t.copy_(torch.exp2(torch.randint(-9, 9, t.shape, generator=g, device="cuda").float()))
    return cache


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _reserve(cache, plain, start, n_new, count=None):
    status = cache.sp_cache_reserve(_i32(start), n_new, None if count is None else _i32(count))
    want = plain.reserve(start, n_new, count)
    assert tuple(status.tolist()) == want
    plain.check(cache)
    return want


def _fork(cache, plain, dst, src=None):
    cache.sp_cache_fork(_i32(dst), None if src is None else _i32(src))
    plain.fork(dst, src)
    plain.check(cache)


@pytest.mark.parametrize("heads,dim,block", [(1, 64, 16), (3, 128, 32), (5, 64, 64), (40, 128, 64)])
def test_answers_of_a_prompt(sp, heads, dim, block):
    cache = _pool(sp, 7, 5, 40, heads, dim, block)
    plain = ref.PlainPages(cache)
    length = [2 * block + 5] + [0] * 6
    _reserve(cache, plain, [0] * 7, length[0], length)
    _fork(cache, plain, list(range(1, 7)), [0] * 6)
    for step in range(3):                                   # own copies at the first, nothing at the others
        _reserve(cache, plain, [length[0] + step] * 7, 1)
    _fork(cache, plain, [2, 5])                             # two have ended
    _fork(cache, plain, [0, 1, 2, 3, 4, 6], [3, 3, 0, 6, 1, 1])   # beams change places
    _reserve(cache, plain, [length[0] + 3] * 5 + [-1] + [length[0] + 3], block + 1)
    live = cache.sp_cache_compact()
    assert live.item() == plain.compact()
    plain.check(cache)


def test_fork_of_rows_named_twice_absent_rows_and_odd_entries(sp):
    cache = _pool(sp, 6, 70, 500)
    plain = ref.PlainPages(cache)
    _reserve(cache, plain, [0, 3, 16, 40, 0, 5], 1100, [1100, 64, 1000, 1, 0, -4])
    cache.table[1, 2], cache.table[1, 9] = 10 ** 6, -7      # name no block: copied as they are
    plain.table[1][2], plain.table[1][9] = 10 ** 6, -7
    _fork(cache, plain, [4, 5, 4, 9, -1, 0], [0, 1, 1, 2, 2, 17])
    _fork(cache, plain, [2], [2])
    _fork(cache, plain, [0, 1, 2, 3, 4, 5], [1, 2, 3, 4, 5, 0])
    cache.sp_cache_fork(_i32([]), _i32([]))
    plain.check(cache)


def test_fork_of_many_rows(sp):
    """More rows than shared memory stages."""
    n = 2000
    cache = _pool(sp, n, 33, 3000, heads=1, seed=3)
    plain = ref.PlainPages(cache)
    _reserve(cache, plain, [0] * n, 16, [16 if b % 3 == 0 else 0 for b in range(n)])
    rng = random.Random(5)
    dst = rng.sample(range(n), n)
    _fork(cache, plain, dst, [rng.randrange(-1, n) for _ in dst])


def test_reserve_in_a_full_pool_changes_nothing(sp):
    cache = _pool(sp, 3, 4, 7)
    plain = ref.PlainPages(cache)
    assert _reserve(cache, plain, [0, 0, 0], 33) == (2, 7)
    assert _reserve(cache, plain, [0, 0, 0], 33, [33, 33, 16]) == (0, 0)
    assert _reserve(cache, plain, [33, 10, 16], 16) == (2, 0)  # places 48 and 16
    assert _reserve(cache, plain, [33, 10, 15], 1) == (0, 0)
    _fork(cache, plain, [0])
    assert _reserve(cache, plain, [0, 33, 16], 10 ** 9, [0, 10 ** 9, 17])[0] == 0


def test_reserve_where_only_some_sharers_ask(sp):
    cache = _pool(sp, 4, 3, 12)
    plain = ref.PlainPages(cache)
    _reserve(cache, plain, [0] * 4, 20, [20, 0, 0, 0])
    _fork(cache, plain, [1, 2, 3], [0, 0, 0])
    _reserve(cache, plain, [20] * 4, 3, [0, 3, 0, 3])       # two of four: both get copies
    _reserve(cache, plain, [23, 0, 20, 0], 1, [1, 0, 1, 0])  # the other two: the first keeps the block
    _reserve(cache, plain, [16, 23, 15, 40], 1)


@pytest.mark.parametrize("n_blocks,n_seqs", [(1, 1), (31, 3), (1024, 9), (5000, 200)])
def test_reserve_and_compact_pools_of_all_sizes(sp, n_blocks, n_seqs):
    """Blocks in use at random; every request of random lengths."""
    rng = random.Random(n_blocks)
    cache = _pool(sp, n_seqs, 30, n_blocks, heads=1, seed=n_blocks)
    plain = ref.PlainPages(cache)
    used = rng.sample(range(n_blocks), n_blocks // 2)
    for i, x in enumerate(used):
        b, place = i % n_seqs, i // n_seqs
        if place < 30:
            plain.table[b][place] = x
            plain.refs[x] = 1
    cache.table.copy_(_i32(plain.table))
    cache.refs.copy_(_i32(plain.refs))
    for _ in range(3):
        _reserve(cache, plain, [rng.randrange(0, 400) for _ in range(n_seqs)], 60, [rng.randrange(-1, 70) for _ in range(n_seqs)])
        rows = [rng.randrange(n_seqs) for _ in range(n_seqs // 2)]
        _fork(cache, plain, rows, [rng.randrange(-1, n_seqs) for _ in rows])
    table, refs = torch.full_like(cache.table, -5), torch.full_like(cache.refs, -5)
    before = ref.PlainPages(cache)
    live = cache.sp_cache_compact(table_out=table, refs_out=refs)
    assert live.item() == plain.compact()
    plain.check(cache, table, refs)
    assert cache.table.tolist() == before.table and cache.refs.tolist() == before.refs
    assert cache.sp_cache_compact(table_out=table, refs_out=refs).item() == live.item()   # the same again
    plain.check(cache, table, refs)


def test_compact_of_empty_full_and_inconsistent_pools(sp):
    cache = _pool(sp, 2, 3, 6)
    plain = ref.PlainPages(cache)
    assert cache.sp_cache_compact().item() == plain.compact() == 0
    plain.check(cache)
    _reserve(cache, plain, [0, 0], 48)
    assert cache.sp_cache_compact().item() == plain.compact() == 6
    plain.check(cache)
    cache.refs[2], plain.refs[2] = 0, 0                     # an entry that names a free block
    cache.refs[4], plain.refs[4] = -2, -2
    cache.table[1, 0], plain.table[1][0] = 77, 77
    assert cache.sp_cache_compact().item() == plain.compact() == 4
    plain.check(cache)


def test_a_wide_table_view_and_rows_behind_it(sp):
    """A table that is part of a wider one: what lies beside it stays."""
    cache = _pool(sp, 5, 4, 20)
    wide = torch.full((5, 9), 123456, dtype=torch.int32, device="cuda")
    wide[:, :4] = -1
    cache = sp.KvCache(cache.k, cache.v, cache.k_scale, cache.v_scale, wide[:, :4], refs=cache.refs)
    plain = ref.PlainPages(cache)
    _reserve(cache, plain, [0] * 5, 40)
    _fork(cache, plain, [0, 1], [4, 4])
    assert cache.sp_cache_compact().item() == plain.compact()
    plain.check(cache)
    assert (wide[:, 4:] == 123456).all()


def test_captured_calls_with_new_values(sp):
    cache = _pool(sp, 4, 6, 40)
    plain = ref.PlainPages(cache)
    dst, src, start = _i32([1, 2, 3]), _i32([0, 0, 0]), _i32([0, 0, 0, 0])
    status, live = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.sp_cache_fork(dst, src)
        cache.sp_cache_reserve(start, 5, status=status)
        cache.sp_cache_compact(live)
    plain.check(cache)
    for values in (([1, 2, 3], [0, 0, 0], [0, 0, 0, 0]), ([0, 1, 2], [3, 0, 0], [3, 7, 15, 30]), ([0, 2, 2], [-1, 1, 3], [20, 5, 17, 47])):
        for t, v in zip((dst, src, start), values):
            t.copy_(_i32(v))
        graph.replay()
        plain.fork(values[0], values[1])
        want = plain.reserve(values[2], 5)
        assert tuple(status.tolist()) == want and live.item() == plain.compact()
        plain.check(cache)


def test_many_rows_of_a_large_pool(sp):
    """32767 rows and 70000 blocks, against the same done with whole tensors."""
    n_seqs, n_blocks, g = 32767, 70000, torch.Generator().manual_seed(9)
    cache = sp.KvCache.pool(n_seqs, 32, n_blocks, 1, 64, 16)
    cache.k.copy_(torch.randint(0, 256, cache.k.shape, generator=g, dtype=torch.uint8))
    cache.v.copy_(torch.randint(0, 256, cache.v.shape, generator=g, dtype=torch.uint8))
    used = torch.randperm(n_blocks, generator=g)[:20000].to(torch.int32)
    table = torch.full((n_seqs, 2), -1, dtype=torch.int32)
    table[torch.randperm(n_seqs, generator=g)[:20000], 0] = used
    count = lambda t: torch.bincount(t[t >= 0].long().flatten(), minlength=n_blocks).to(torch.int32)
    cache.table.copy_(table)
    cache.refs.copy_(count(table))
    # a row without a first block gets a free one, in the order of the rows
    status = cache.sp_cache_reserve(torch.zeros(n_seqs, dtype=torch.int32, device="cuda"), 16)
    free = torch.nonzero(count(table) == 0).flatten().to(torch.int32)
    wants = table[:, 0] < 0
    table[wants, 0] = free[:int(wants.sum())]
    assert torch.equal(cache.table.cpu(), table) and torch.equal(cache.refs.cpu(), count(table))
    assert status.tolist() == [0, n_blocks - n_seqs]
    # rows change places
    dst = torch.randperm(n_seqs, generator=g)[:20000].to(torch.int32)
    src = torch.randint(-1, n_seqs, (20000,), generator=g, dtype=torch.int32)
    cache.sp_cache_fork(dst.cuda(), src.cuda())
    rows = torch.cat([table, torch.full((1, 2), -1, dtype=torch.int32)])   # the last one for -1
    table[dst.long()] = rows[src.long()]
    assert torch.equal(cache.table.cpu(), table) and torch.equal(cache.refs.cpu(), count(table))
    # the same contents at the front of the pool
    old_k, old_v, old = cache.k.cpu(), cache.v.cpu(), count(table)
    n = cache.sp_cache_compact().item()
    assert n == int((old > 0).sum())
    new = cache.table.cpu()
    named = table >= 0
    assert torch.equal(new >= 0, named) and int(new.max()) < n and torch.equal(cache.refs.cpu(), count(new))
    assert torch.equal(cache.k.cpu()[new[named].long()], old_k[table[named].long()])
    assert torch.equal(cache.v.cpu()[new[named].long()], old_v[table[named].long()])
    low = named & (table < n)
    assert torch.equal(new[low], table[low])                                # those numbered below n stay
