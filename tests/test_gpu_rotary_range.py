"""Norms of rows whose squares binary32 does not hold, against the definition in binary64."""
import numpy as np
import pytest
import torch

from . import answers_reference as ref
from .test_gpu_rotary import _freq, sp  # noqa: F401

pytestmark = pytest.mark.gpu


def _check(got, x, w, start, freq, pairs, eps):
    """As for ordinary rows (half a step of the output, 32 roundings of 2^-24 of what a value is made of:
    24 of them there, of the powers of two here only a factor of 2^-126 may lose two bits), and half of
    bf16's least step."""
    want, mag = ref.norm_rotary(x, w, start, freq, pairs, eps)
    got = got.double().cpu().numpy()
    far = ~(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -134 + 32 * 2.0 ** -24 * mag)
    assert not far.any(), (np.argwhere(far)[:3], got[far][:3], want[far][:3])


@pytest.mark.parametrize("eps", [0.0, 1e-35, 1e-6])
@pytest.mark.parametrize("dim,rotary,pairs", [(64, 64, False), (64, 32, True), (128, 128, True), (128, 128, False), (128, 24, False), (80, 40, False), (256, 0, False)])
def test_large_and_small_rows(sp, dim, rotary, pairs, eps):  # noqa: F811
    """bf16 rows of 2^-126 to 2^125, alone and with one value far above the others."""
    g = torch.Generator().manual_seed(dim)
    powers = [-126, -120, -90, -64, -60, -40, 0, 40, 60, 63, 64, 90, 120, 125]
    x = torch.randn(len(powers), 3, 3, dim, generator=g, dtype=torch.float64).clamp(-3, 3)
    x = (x * 2.0 ** torch.tensor(powers, dtype=torch.float64)[:, None, None, None])
    x[:, 1, :, 5] *= 2.0 ** -30
    x[:6, 2, 0, dim - 3] = 2.0 ** 70
    x = x.to(torch.bfloat16)
    w = torch.randn(dim, generator=g).to(torch.bfloat16)
    freq, start = _freq(rotary), list(range(len(powers)))
    q, k = sp.sp_qk_norm_rotary(x.cuda(), x.cuda()[:, :, :1], torch.tensor(start, dtype=torch.int32).cuda(), freq.cuda(),
                                q_weight=w.cuda(), k_weight=w.cuda(), eps=eps, pairs=pairs)
    eps = float(np.float32(eps))
    _check(q, x, w, start, freq, pairs, eps)
    _check(k, x[:, :, :1], w, start, freq, pairs, eps)


@pytest.mark.parametrize("dim,pairs", [(64, False), (128, True), (80, False)])
def test_rows_that_are_not_finite_or_zero(sp, dim, pairs):  # noqa: F811
    """An infinity under the norm becomes NaN and the others 0; a NaN takes its row; a row of zeros without eps is NaN."""
    x = torch.randn(4, 1, 2, dim, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    x[0, 0, 0, 7], x[1, 0, 1, 3], x[2] = float("inf"), float("nan"), 0.0
    x[3, 0, 0] *= 2.0 ** 100
    x[3, 0, 0, 1] = float("-inf")
    w, none = torch.ones(dim, dtype=torch.bfloat16), torch.zeros(0)
    q, _ = sp.sp_qk_norm_rotary(x.cuda(), x.cuda()[:, :, :0], torch.zeros(4, dtype=torch.int32).cuda(), none.cuda(), q_weight=w.cuda(), eps=0.0, pairs=pairs)
    want, _ = ref.norm_rotary(x, w, [0] * 4, none, pairs, 0.0)
    q = q.double().cpu().numpy()
    assert np.array_equal(np.isnan(q), np.isnan(want))
    ok = ~np.isnan(want)
    assert (np.abs(q - want)[ok] <= 2.0 ** -8 * np.abs(want)[ok] + 32 * 2.0 ** -24 * np.abs(want)[ok]).all()
