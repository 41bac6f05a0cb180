"""Attention over the 8-bit cache where the roundings of its weights and queries show in the output."""
import numpy as np
import pytest
import torch

from . import serve_reference as ref
from .test_gpu_cache import _check_attention, _filled

pytestmark = pytest.mark.gpu

DTYPES = [torch.float16, torch.bfloat16]
UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}    # half the spacing at 1
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}  # half the smallest subnormal


@pytest.fixture(scope="module")
def sp():
    from paper_2501_16376_b200 import binding
    yield binding
    assert binding.sp_wait_status() == 0


def _attention(sp, K, V, Q, max_len=None):
    """Own and binary64 results, and the weighted magnitudes of the values; scale 1."""
    B, L, H, D = K.shape
    cache = sp.KvCache.empty(B, L, H, D, 32)
    cache.sp_cache_append(K.cuda(), V.cuda(), torch.zeros(B, dtype=torch.int32, device="cuda"))
    lens = torch.full((B,), L, dtype=torch.int32, device="cuda")
    got = cache.sp_cache_attention(Q.cuda(), lens, max_len or L, scale=1.0).cpu().double().numpy()
    want, _, _, mag, _ = ref.PlainCache(cache).attention(Q, [L] * B, max_len or L, 1.0)
    return got, want, mag


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,group,D", [(4, 1, 64), (2, 8, 128), (1, 16, 128)])
def test_values_that_cancel(sp, heads, group, D, dtype):
    """Eight tokens with values of 1 and -1: some outputs are far smaller than what they are made
    of, so that the weights' own errors are seen.  Scores are one product of at most 1, so a weight
    is off by a few units of 2^-23 (the score's factor, the exponential) and 2^-22 (two binary16
    parts), the sums of eight by as much again: 2^-19 of the values' weighted magnitudes."""
    B, L = 16, 8
    g = torch.Generator().manual_seed(D + group)
    K = torch.zeros(B, L, heads, D)
    K[..., 0] = torch.rand(B, L, heads, generator=g)
    V = torch.randint(0, 2, (B, L, heads, D), generator=g) * 2.0 - 1.0
    Q = torch.zeros(B, 1, heads * group, D)
    Q[..., 0] = torch.rand(B, 1, heads * group, generator=g)
    got, want, mag = _attention(sp, K.to(dtype), V.to(dtype), Q.to(dtype))
    err = np.abs(got - want)
    assert (err <= UNIT[dtype] * np.abs(want) + 2.0 ** -19 * mag + TINY[dtype]).all(), (err - UNIT[dtype] * np.abs(want)).max()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("L,heads,D", [(200, 4, 64), (3000, 1, 128), (20000, 2, 64)])
@pytest.mark.parametrize("below", [18.0, 24.0, 26.0])
def test_outputs_that_lie_in_many_small_weights(sp, L, heads, D, below, dtype):
    """One token takes nearly all the attention and has the value 0 (a sink), so that the output is
    made of weights 2^-26, 2^-34.6 and 2^-37.5 of the largest.  A score is one exact product of at most
    26, times log2(e) in binary32: its exponent is off by 2^-18 at most (38 * 2^-24, and the
    exponential's own 2^-22), a weight by as much of itself; the two parts end 2^-37 below weights
    of at least 2^7, 2^-44 relative to the largest, and the sums in binary32 lose 2^-24 for each of
    a lane's additions, L / 16 at most."""
    g = torch.Generator().manual_seed(L)
    K = torch.zeros(1, L, heads, D)
    K[..., 0] = -below
    top = 448.0 * (64 if dtype == torch.float16 else 1)
    V = (torch.rand(1, L, heads, D, generator=g) * 0.9 + 0.1) * top
    at = L // 3
    K[:, at, :, 0], V[:, at] = 0.0, 0.0
    Q = torch.zeros(1, 2, heads * 2, D)
    Q[..., 0] = 1.0
    got, want, mag = _attention(sp, K.to(dtype), V.to(dtype), Q.to(dtype))
    assert (want > 1e-9).all()
    err = np.abs(got - want)
    allowed = (UNIT[dtype] * want + (2.0 ** -17 + L / 16 * 2.0 ** -24) * mag
               + L * 2.0 ** -44 * top + TINY[dtype])
    assert (err <= allowed).all(), (err / allowed).max()


@pytest.mark.parametrize("heads,group,n_q,D", [(2, 1, 1, 64), (1, 4, 1, 128), (1, 8, 1, 128), (2, 4, 3, 64)])
@pytest.mark.parametrize("far", [20, 34, 45, 60])
def test_queries_with_a_channel_far_above_the_others(sp, heads, group, n_q, D, far):
    """bf16 queries, one channel of which is 2^far times the others and meets keys of 0: the others alone
    make the scores.  They are held to 2^-20 of themselves at least (eight bits of bf16, exact, or two
    binary16 parts), so a score of D / 16 sums is off as in any other row: (D / 16 + 4) * 2^-22 of its terms'
    magnitudes, and a weight by twice that."""
    B, L = 2, 150
    g = torch.Generator().manual_seed(far)
    K, V = torch.randn(2, B, L, heads, D, generator=g)
    Q = torch.randn(B, n_q, heads * group, D, generator=g) * 0.3
    K[..., 11] = 0
    Q[..., 11] = 2.0 ** far
    Q[0, 0, 0] = torch.randn(D, generator=g)                   # one ordinary row
    K, V, Q = K.bfloat16(), V.bfloat16(), Q.bfloat16()
    cache = sp.KvCache.empty(B, L, heads, D, 32)
    cache.sp_cache_append(K.cuda(), V.cuda(), torch.zeros(B, dtype=torch.int32, device="cuda"))
    lens = torch.full((B,), L, dtype=torch.int32, device="cuda")
    lse = torch.zeros(B, n_q, heads * group, device="cuda")
    got = cache.sp_cache_attention(Q.cuda(), lens, L, scale=1.0, lse=lse).cpu().double().numpy()
    want, want_lse, _, mag, terms = ref.PlainCache(cache).attention(Q, [L] * B, L, 1.0)
    d = (D / 16 + 4) * 2.0 ** -22 * terms + 2.0 ** -21
    assert d.max() < 0.001
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + (4 * d[..., None] + 2.0 ** -20) * mag).all()
    assert (np.abs(lse.cpu().double().numpy() - want_lse) <= 2 * d + 2.0 ** -20 * np.abs(want_lse)).all()


@pytest.mark.parametrize("lens,heads,group,n_q,D", [([3000, 700], 2, 4, 1, 128), ([40, 16, 0, 2], 1, 2, 4, 128),
                                                    ([900, 20], 1, 8, 3, 64), ([5000], 1, 1, 1, 64)])
def test_such_queries_in_every_way_a_call_ends(sp, lens, heads, group, n_q, D):
    """Clusters and joined splits, accumulated weights, and NaN among the call's own tokens."""
    cache = _filled(sp, lens, heads, D, 16, dtype=torch.bfloat16)
    at = torch.arange(cache.k.numel(), device="cuda").view_as(cache.k) % D == 7
    cache.k[at] = 0
    for b, n in enumerate(lens):
        if n_q > 1 and n > 2:
            cache.v[int(cache.table[b, (n - 1) // 16]), 0, (n - 1) % 16, 5] = 0x7f
    Q = torch.randn(len(lens), n_q, heads * group, D, generator=torch.Generator().manual_seed(1))
    Q[:, :, ::2, 7] = 2.0 ** 50
    acc_in = torch.rand(len(lens), heads, max(lens), generator=torch.Generator().manual_seed(1)).cuda()
    _check_attention(sp, cache, Q.bfloat16(), lens, max(lens), acc_in=acc_in)
