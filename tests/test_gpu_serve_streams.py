"""Serving calls on the current stream and on another in turn, nothing synchronised in between: every
call leaves the bits that it leaves alone, whatever memory the allocator reuses."""
import pytest
import torch

from . import serve_reference as ref
from .test_gpu_cache import _filled, _i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2501_16376_b200 import binding
    yield binding
    assert binding.sp_wait_status() == 0


def _alternate(call, n=24):
    """call(i, stream) -> tensors, without regard to the stream it runs on."""
    want = [[t.clone() for t in call(i, None)] for i in range(2)]
    torch.cuda.synchronize()
    side, got = torch.cuda.Stream(), []
    for i in range(n):
        outs = call(i % 2, None)
        if i % 3 == 0:
            got.append((i % 2, outs))
        del outs                                       # its memory, and the scratch, are free at once
        outs = call((i + 1) % 2, side)
        if i % 4 == 0:
            got.append(((i + 1) % 2, outs))
        del outs
    torch.cuda.synchronize()
    for i, outs in got:
        assert all(torch.equal(a, b) for a, b in zip(outs, want[i]))


@pytest.mark.parametrize("mode,T", [(0, 3), (0, 300), (1, 300), (1, 2000)])
def test_products(sp, mode, T):
    codes, scales, _ = ref.mx4_random(1000, 2051, 3)
    codes, scales = codes.cuda(), scales.cuda()
    X = [torch.randn(T, 2051, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda() for i in range(2)]
    _alternate(lambda i, stream: [sp.sp_mx4_linear(X[i], codes, scales, mode, stream=stream)])


def test_quantisation(sp):
    W = [torch.randn(700, 2048, generator=torch.Generator().manual_seed(i)).half().cuda() for i in range(2)]

    def call(i, stream):
        codes, scales = sp.sp_mx4_quantize(W[i], stream=stream)
        return codes, scales, sp.sp_mx4_dequantize(codes, scales, 2048, stream=stream)
    _alternate(call)


@pytest.mark.parametrize("lens", [[300, 290], [6000, 5000]])
def test_attention_and_eviction(sp, lens):
    cache = _filled(sp, lens, 2, 128, 32)
    Q = [torch.randn(2, 1, 8, 128, generator=torch.Generator().manual_seed(i)).half().cuda() for i in range(2)]
    n, L = _i32(*lens), lens[0]
    acc = [torch.zeros(2, 2, L, device="cuda") for _ in range(2)]
    old = [torch.rand(2, 2, L, generator=torch.Generator().manual_seed(i)).cuda() for i in range(2)]
    dst = [sp.KvCache.empty(2, 128, 2, 128, 32) for _ in range(2)]

    def call(i, stream):
        # the accumulated weights, and the cache evicted into, are the caller's: one for each stream
        at = 0 if stream is None else 1
        O = cache.sp_cache_attention(Q[i], n, L, acc_out=acc[at], stream=stream)
        return (O, *cache.sp_cache_evict(n, L, old[i], 100, 9, dst[at], stream=stream))
    _alternate(call)


def test_attention_over_many_splits_with_a_query_for_every_stream(sp):
    cache = _filled(sp, [9000], 1, 64, 16)
    Q = [torch.randn(1, 3, 4, 64, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda() for i in range(2)]
    n = _i32(9000)
    _alternate(lambda i, stream: [cache.sp_cache_attention(Q[i], n, 9000, stream=stream)])
