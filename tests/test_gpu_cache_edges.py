"""The 8-bit key/value cache at its edges: zeros from blocks of large values, no queries, huge scores."""
import numpy as np
import pytest
import torch

from . import serve_reference as ref
from .test_gpu_cache import _check_attention, _check_evict, _filled, _i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2501_16376_b200 import binding
    yield binding
    assert binding.sp_wait_status() == 0


@pytest.mark.parametrize("dim,block", [(64, 16), (128, 32), (128, 64)])
@pytest.mark.parametrize("kept", [1, 16, 40])
def test_evicted_zeros_stay_zeros(sp, dim, block, kept):
    """Zero tokens of blocks whose scale is large (their largest value is left behind) are kept alone,
    beside NaN, and beside tiny values: results are equal to the definition's, bit for bit."""
    L, heads = 200, 3
    g = torch.Generator().manual_seed(kept)
    K, V = torch.zeros(2, 1, L, heads, dim)
    K[0, ::8, 0], V[0, ::8, 0] = 2000.0, -3e4                       # scales of 8 and 128
    K[0, ::8, 1], V[0, ::8, 1] = torch.randn(dim, generator=g) * 1e3, 6e4
    V[0, 1::4, 1, ::5] = float("nan")
    K[0, ::8, 2], V[0, 2::4, 2] = 1.0, 2.0 ** -24
    V[0, ::8, 2] = 448.0
    cache = sp.KvCache.empty(1, L, heads, dim, block)
    cache.sp_cache_append(K.half().cuda(), V.half().cuda(), _i32(0))
    acc = torch.rand(1, heads, L, generator=g)
    acc[..., ::8] = 0.0                                             # the large ones go
    _check_evict(sp, cache, [L], L, acc, kept, 0)
    # bf16 holds values large enough that the factor between two scales passes binary32's range
    K[0, ::8], V[0, ::8] = 1e38, -3e38
    V[0, 3::4, 0, 7] = 1e-38
    cache = sp.KvCache.empty(1, L, heads, dim, block)
    cache.sp_cache_append(K.bfloat16().cuda(), V.bfloat16().cuda(), _i32(0))
    _check_evict(sp, cache, [L], L, acc, kept, 0)


def test_attention_after_the_eviction_of_zeros(sp):
    K, V = torch.zeros(2, 1, 16, 1, 64)
    K[0, 0], V[0, 0] = 1e4, 1e4
    cache, dst = sp.KvCache.empty(1, 32, 1, 64, 16), sp.KvCache.empty(1, 8, 1, 64, 16)
    cache.sp_cache_append(K.half().cuda(), V.half().cuda(), _i32(0))
    kept, _, lens = cache.sp_cache_evict(_i32(16), 16, torch.zeros(1, 1, 16, device="cuda"), 8, 8, dst)
    assert kept.flatten().tolist() == list(range(8, 16))
    O = dst.sp_cache_attention(torch.ones(1, 1, 1, 64, dtype=torch.float16, device="cuda"), lens, 8)
    assert np.array_equal(O.cpu().numpy(), np.zeros((1, 1, 1, 64)))


@pytest.mark.parametrize("in_place", [False, True])
def test_no_query_leaves_the_accumulated_weights(sp, in_place):
    """What the definition gives for n_q = 0: acc_in up to the length, 0 past it."""
    lens, L = [1500, 0, 70, 2000, -3], 1600
    cache = sp.KvCache.empty(5, 1600, 2, 64, 16)
    acc = torch.rand(5, 2, L, generator=torch.Generator().manual_seed(0))
    want = acc.clone()
    for b, n in enumerate(lens):
        want[b, :, max(n, 0):] = 0
    Q = torch.zeros(5, 0, 4, 64, dtype=torch.float16, device="cuda")
    acc_in = acc.cuda()
    acc_out = acc_in if in_place else torch.full_like(acc_in, 7.0)
    O = cache.sp_cache_attention(Q, _i32(*lens), L, acc_in=acc_in, acc_out=acc_out)
    assert O.shape == Q.shape and torch.equal(acc_out.cpu(), want)
    cache.sp_cache_attention(Q, _i32(*lens), L, acc_out=acc_out)
    assert (acc_out == 0).all()
    cache.sp_cache_attention(Q, _i32(*lens), 0, acc_out=acc_out)
    cache.sp_cache_attention(Q, _i32(*lens), L)


@pytest.mark.parametrize("group,n_q", [(1, 1), (2, 1), (3, 1), (4, 1), (8, 1), (4, 4)])
@pytest.mark.parametrize("L", [40, 3000])
@pytest.mark.parametrize("score", [300.0, -2.0 ** 16, 2.0 ** 24])
def test_accumulated_weights_of_large_scores(sp, L, score, group, n_q):
    """Equal scores of any size give every token its share, whatever the size: the scores are one exact
    product, equal for all tokens, so a weight is off by the roundings of its exponential and of the
    sum of up to 3000 equal terms (below 2^-14 of itself; few are added one by one in binary32)."""
    K = torch.zeros(2, L, 2, 64)
    K[..., 9] = 2.0
    Q = torch.zeros(2, n_q, 2 * group, 64)
    Q[..., 9] = score / 2
    cache = sp.KvCache.empty(2, L, 2, 64, 16)
    cache.sp_cache_append(K.bfloat16().cuda(), K.bfloat16().cuda(), _i32(0, 0))
    acc = torch.zeros(2, 2, L, device="cuda")
    cache.sp_cache_attention(Q.bfloat16().cuda(), _i32(L, L), L, scale=1.0, acc_out=acc)
    want = np.zeros(L)
    for i in range(n_q):
        end = L - n_q + i + 1
        want[:end] += group / end
    assert (np.abs(acc.cpu().double().numpy() / want - 1) <= 2.0 ** -14).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,group,n_q,lens", [(2, 4, 34, [200, 33, 5]), (1, 1, 129, [129, 300]), (1, 5, 103, [400]),
                                                  (1, 1, 8192, [700])])
def test_many_query_rows(sp, heads, group, n_q, lens, dtype):
    cache = _filled(sp, lens, heads, 64, 16)
    Q = torch.randn(len(lens), n_q, heads * group, 64, generator=torch.Generator().manual_seed(n_q)).to(dtype)
    acc_in = torch.rand(len(lens), heads, max(lens), generator=torch.Generator().manual_seed(1)).cuda()
    _check_attention(sp, cache, Q, lens, max(lens), acc_in=acc_in)


@pytest.mark.parametrize("L", [1, 20, 3000])
@pytest.mark.parametrize("size", [1e15, 1e18])
def test_scores_of_any_finite_size_are_scores(sp, L, size):
    """Queries and keys whose products are far below any ordinary score (-1e30, -1e36, equal for all
    tokens): the weights are 1 / L all the same, and lse is the score."""
    g = torch.Generator().manual_seed(L)
    K, V = torch.zeros(1, L, 2, 64), torch.randn(1, L, 2, 64, generator=g)
    K[..., 3] = -size
    Q = torch.zeros(1, 1, 4, 64)
    Q[..., 3] = size
    K, V, Q = K.bfloat16(), V.bfloat16(), Q.bfloat16()
    cache = sp.KvCache.empty(1, L, 2, 64, 32)
    cache.sp_cache_append(K.cuda(), V.cuda(), _i32(0))
    stored = ref.PlainCache(cache)
    score = stored.dense("k", 0, 0, 1)[0][0, 3] * float(Q[0, 0, 0, 3])
    lse, acc = torch.zeros(1, 1, 4, device="cuda"), torch.zeros(1, 2, L, device="cuda")
    for out in (acc, None):
        O = cache.sp_cache_attention(Q.cuda(), _i32(L), L, scale=1.0, lse=lse, acc_out=out).cpu().double()
        # weights 1/L, sums in binary32 and one rounding to bf16
        want = np.stack([stored.dense("v", 0, h // 2, L)[0].mean(0) for h in range(4)])
        mag = np.stack([np.abs(stored.dense("v", 0, h // 2, L)[0]).mean(0) for h in range(4)])
        assert (np.abs(O.numpy()[0, 0] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -17 * mag).all()
        assert np.abs(lse.cpu().double().numpy() / score - 1).max() <= 2.0 ** -20
    assert (acc.cpu() * L / 2 - 1).abs().max() <= 2.0 ** -17


def test_captured_cache_calls_leave_the_same_bits(sp):
    """A decoding step of append, attention and eviction in one graph: lengths are read on the device."""
    B, L, H, D = 2, 600, 2, 128
    g = torch.Generator().manual_seed(0)
    K, V = (torch.randn(B, L, H, D, generator=g).half().cuda() for _ in range(2))
    k, v, q = (torch.randn(B, 1, n, D, generator=g).half().cuda() for n in (H, H, 4 * H))
    start, lens = _i32(500, 30), _i32(501, 31)

    def fresh():
        cache = sp.KvCache.empty(B, 640, H, D, 32)
        cache.sp_cache_append(K, V, _i32(0, 0))
        return cache, sp.KvCache.empty(B, 64, H, D, 32), torch.zeros(B, H, 640, device="cuda")

    def step(cache, dst, acc):
        cache.sp_cache_append(k, v, start)
        O = cache.sp_cache_attention(q, lens, 640, acc_in=acc, acc_out=acc)
        return (O, *cache.sp_cache_evict(lens, 640, acc, 64, 4, dst), dst.k, dst.v, dst.k_scale, dst.v_scale)
    a, b = fresh(), fresh()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(*b)
    for _ in range(3):
        want = [t.clone() for t in step(*a)]
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(want, outs))
        start += 1
        lens += 1
