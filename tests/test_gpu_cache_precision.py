"""Attention over the 8-bit cache where the roundings of its weights show in the output."""
import numpy as np
import pytest
import torch

from . import serve_reference as ref

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
