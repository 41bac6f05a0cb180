"""Norms and positions of queries and keys against their definition in binary64."""
import numpy as np
import pytest
import torch

from . import answers_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = [torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def sp():
    from paper_2501_16376_b200 import binding
    return binding


def _freq(rotary, theta=10000.0):
    return (theta ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / max(rotary, 1))).float()


def _check(got, x, w, start, freq, pairs, eps):
    """Half a step of the output (at least half of binary16's least step), and 32 roundings of 2^-24 of
    what a value is made of: the sum of squares (a tree of at most 256 terms: 16 of them in a lane, so
    up to 19 roundings, halved by the root), root, weight, cosine (its angle rounded to 2^-25 of a
    half turn: 4), products and sum."""
    want, mag = ref.norm_rotary(x, w, start, freq, pairs, eps)
    got = got.double().cpu().numpy()
    dtype = x.dtype
    bound = torch.finfo(dtype).eps / 2 * np.abs(want) + 2.0 ** -25 * (dtype == torch.float16) + 32 * 2.0 ** -24 * mag
    assert np.array_equal(np.isnan(got), np.isnan(want))
    far = np.abs(got - want) > bound
    assert not far.any(), (np.argwhere(far)[:3], got[far][:3], want[far][:3])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dim,rotary", [(64, 64), (128, 128), (64, 16), (128, 48), (128, 20), (64, 0), (80, 80), (256, 64), (2, 2), (6, 4)])
def test_against_the_definition(sp, dim, rotary, pairs, dtype):
    g = torch.Generator().manual_seed(dim + rotary)
    for B, n, H, Hk, norm, start in ((1, 1, 5, 1, True, [7]), (3, 13, 4, 2, False, [0, 1000, 2 ** 30]), (2, 5, 40, 8, True, [-3, 10 ** 6])):
        Q, K = (torch.randn(B, n, h, dim, generator=g).mul_(2).to(dtype) for h in (H, Hk))
        wq, wk = ((torch.randn(dim, generator=g)).to(dtype) if norm else None for _ in range(2))
        freq = _freq(rotary)
        dev = lambda t: None if t is None else t.cuda()
        q, k = sp.sp_qk_norm_rotary(Q.cuda(), K.cuda(), torch.tensor(start, dtype=torch.int32).cuda(), freq.cuda(),
                                    q_weight=dev(wq), k_weight=dev(wk), eps=1e-5, pairs=pairs)
        _check(q, Q, wq, start, freq, pairs, 1e-5)
        _check(k, K, wk, start, freq, pairs, 1e-5)


@pytest.mark.parametrize("n", [1, 149, 1300])
def test_many_tokens_in_place_and_from_views(sp, n):
    """Views of one projection's output, turned where they lie; what lies between stays as it was."""
    g = torch.Generator().manual_seed(n)
    x = torch.randn(2, n, 3 + 2 + 2, 64, generator=g).to(torch.bfloat16)
    d, freq, start = x.cuda(), _freq(64), [5, 99]
    sp.sp_qk_norm_rotary(d[:, :, :3], d[:, :, 3:5], torch.tensor(start, dtype=torch.int32).cuda(), freq.cuda(),
                         Q_out=d[:, :, :3], K_out=d[:, :, 3:5])
    _check(d[:, :, :3], x[:, :, :3], None, start, freq, False, 0.0)
    _check(d[:, :, 3:5], x[:, :, 3:5], None, start, freq, False, 0.0)
    assert torch.equal(d[:, :, 5:].cpu(), x[:, :, 5:])


@pytest.mark.parametrize("offset,dim", [(1, 64), (0, 66)])
def test_unaligned_and_transposed(sp, offset, dim):
    g = torch.Generator().manual_seed(4)
    x = torch.randn(2, 4, 9, dim + 3, generator=g).to(torch.float16)     # heads before tokens
    d, freq, start = x.cuda(), _freq(32), [3, 4]
    w = torch.randn(dim + 1, generator=g).to(torch.float16)
    cut = lambda t: t[:, :, :, offset:offset + dim].transpose(1, 2)
    q, k = sp.sp_qk_norm_rotary(cut(d), cut(d)[:, :, :1], torch.tensor(start, dtype=torch.int32).cuda(), freq.cuda(),
                                q_weight=w.cuda()[1:], pairs=True)
    _check(q, cut(x), w[1:], start, freq, True, 1e-6)
    _check(k, cut(x)[:, :, :1], None, start, freq, True, 1e-6)


def test_broadcast_input_and_no_keys(sp):
    g = torch.Generator().manual_seed(5)
    x = torch.randn(1, 1, 1, 128, generator=g).to(torch.bfloat16)
    Q, d, freq = x.expand(3, 7, 4, 128), x.cuda().expand(3, 7, 4, 128), _freq(128)
    start = [0, 50, 3]
    q, k = sp.sp_qk_norm_rotary(d, d[:, :, :0], torch.tensor(start, dtype=torch.int32).cuda(), freq.cuda())
    _check(q, Q, None, start, freq, False, 0.0)
    assert k.shape == (3, 7, 0, 128)


@pytest.mark.parametrize("dim", [64, 128, 96])
@pytest.mark.parametrize("pairs", [False, True])
def test_what_is_not_finite_stays_in_its_pair(sp, dim, pairs):
    """Without a norm an infinity reaches the value it is turned with, and no other."""
    g = torch.Generator().manual_seed(6)
    x = torch.randn(1, 2, 3, dim, generator=g).to(torch.float16)
    rotary = 32
    x[0, 0, 0, dim - 1], x[0, 1, 2, dim - 8], x[0, 0, 1, 3] = float("inf"), float("nan"), float("nan")
    freq = _freq(rotary)
    q, _ = sp.sp_qk_norm_rotary(x.cuda(), x.cuda()[:, :, :0], torch.tensor([1], dtype=torch.int32).cuda(), freq.cuda(), pairs=pairs)
    q = q.cpu()
    assert q[0, 0, 0, dim - 1] == float("inf") and torch.isnan(q[0, 1, 2, dim - 8])
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[0, 0, 0, dim - 1] = bad[0, 1, 2, dim - 8] = bad[0, 0, 1, 3] = bad[0, 0, 1, 2 if pairs else 3 + rotary // 2] = True
    assert torch.equal(~torch.isfinite(q), bad)


def test_zero_and_largest_rows(sp):
    """A row of zeros stays 0 under its norm; the squares of binary16's largest values fit."""
    x = torch.zeros(1, 2, 2, 64, dtype=torch.float16)
    x[0, 1] = 65504.0
    w, freq = torch.ones(64, dtype=torch.float16), _freq(64)
    q, _ = sp.sp_qk_norm_rotary(x.cuda(), x.cuda()[:, :, :0], torch.tensor([0], dtype=torch.int32).cuda(), freq.cuda(), q_weight=w.cuda(), eps=0.25)
    _check(q, x, w, [0], freq, False, 0.25)


def test_far_places(sp):
    """Places up to 2^31 - 1 + tokens: the angle is worked out in binary64 (2^-24 of a turn there, so
    2^-21.3 of what a value is made of: eight of the roundings allowed)."""
    g = torch.Generator().manual_seed(8)
    Q = torch.randn(2, 3, 2, 64, generator=g).to(torch.float16)
    freq, start = _freq(64), [2 ** 31 - 1, -2 ** 31]
    q, _ = sp.sp_qk_norm_rotary(Q.cuda(), Q.cuda()[:, :, :1], torch.tensor(start, dtype=torch.int32).cuda(), freq.cuda())
    _check(q, Q, None, start, freq, False, 0.0)


def test_captured(sp):
    g = torch.Generator(device="cuda").manual_seed(9)
    Q, K = (torch.randn(2, 3, h, 128, generator=g, device="cuda").to(torch.bfloat16) for h in (8, 2))
    start, freq = torch.tensor([1, 2], dtype=torch.int32).cuda(), _freq(128).cuda()
    q, k = sp.sp_qk_norm_rotary(Q, K, start, freq)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q2, k2 = sp.sp_qk_norm_rotary(Q, K, start, freq)
    start.add_(5)
    graph.replay()
    q, k = sp.sp_qk_norm_rotary(Q, K, start, freq)
    assert torch.equal(q, q2) and torch.equal(k, k2)


@pytest.mark.parametrize("B,n,H,Hk,dim,rotary,pairs,norm", [
    (3, 2501, 3, 1, 64, 64, True, "qk"),       # a block: several tokens at a time, and several turns of them
    (7, 601, 1, 0, 64, 32, False, "q"),
    (2, 1003, 20, 1, 128, 24, False, "k"),     # more heads than a block has threads for, pieces of four
    (1, 2222, 43, 2, 128, 128, False, "qk"),   # more heads, pieces of eight
    (2, 40, 130, 30, 64, 40, True, ""),        # few tokens, heads shared out
])
def test_tokens_and_heads_of_a_block(sp, B, n, H, Hk, dim, rotary, pairs, norm):
    g = torch.Generator().manual_seed(H)
    Q, K = (torch.randn(B, n, h, dim, generator=g).to(torch.bfloat16) for h in (H, Hk))
    wq, wk = ((1 + 0.3 * torch.randn(dim, generator=g)).to(torch.bfloat16) if x in norm else None for x in "qk")
    start, freq = [11 * b for b in range(B)], _freq(rotary)
    dev = lambda t: None if t is None else t.cuda()
    q, k = sp.sp_qk_norm_rotary(Q.cuda(), K.cuda(), torch.tensor(start, dtype=torch.int32).cuda(), freq.cuda(), q_weight=dev(wq),
                                k_weight=dev(wk), pairs=pairs)
    _check(q, Q, wq, start, freq, pairs, 1e-6)
    _check(k, K, wk, start, freq, pairs, 1e-6)
