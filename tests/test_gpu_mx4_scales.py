"""Products of binary16 activations with 4-bit rows whose scales lie far apart: the small weights make
the result where the activations of the large ones are zero."""
import numpy as np
import pytest
import torch

from . import serve_reference as ref
from .test_gpu_mx4 import _check_product, _product_bound

pytestmark = pytest.mark.gpu

SPANS = [0, 30, 35, 36, 37, 38, 40, 60, 110]      # binary orders between a row's scales; 36 fit binary16


@pytest.fixture(scope="module")
def sp():
    from paper_2501_16376_b200 import binding
    yield binding
    assert binding.sp_wait_status() == 0


def _far_apart(rows, cols, T, seed):
    """Codes, scale bytes and activations: blocks 0, 3, 6, ... of row r have a scale 2^SPANS[r % 9] times
    that of the others, and meet zeros."""
    g = np.random.RandomState(seed)
    nb = (cols + 31) // 32
    code = g.randint(0, 16, (rows, nb, 32))
    if cols % 32:
        code[:, -1, cols % 32:] = 0
    byte = np.full((rows, nb), 127 - 28)
    byte[:, ::3] += np.array(SPANS)[np.arange(rows) % len(SPANS), None]
    X = torch.randn(T, cols, generator=torch.Generator().manual_seed(seed)) * 2.0 ** 11
    X.view(-1)[torch.arange(T * cols) % cols // 32 % 3 == 0] = 0
    return code, byte, X.half()


# one tile shared by eight blocks, by few, by none; several tiles of a block, more than eight of them
@pytest.mark.parametrize("T", [1, 8, 9, 40, 150])
@pytest.mark.parametrize("rows,cols", [(40, 4096), (200, 1030), (140, 130), (129, 96), (3, 14336)])
def test_small_weights_count(sp, rows, cols, T):
    code, byte, X = _far_apart(rows, cols, T, rows + T)
    codes, scales = (torch.from_numpy(a) for a in ref.mx4_pack(code, byte))
    V = torch.from_numpy(ref.mx4_values(code, byte)[:, :cols])
    assert (X.double() @ V.t()).abs().median() > 2.0 ** -14          # ordinary binary16 numbers
    _check_product(sp, X, codes, scales, V, sp.SP_MX4_A16)


@pytest.mark.parametrize("rows,cols,T", [(20000, 96, 20), (40000, 96, 700), (19000, 260, 260)])
def test_small_weights_count_in_every_tile_of_a_block(sp, rows, cols, T):
    code, byte, X = _far_apart(rows, cols, T, T)
    byte[np.arange(rows) % 500 != 37, ::3] = 127 - 28                 # a wide row here and there
    codes, scales = (torch.from_numpy(a) for a in ref.mx4_pack(code, byte))
    _check_product(sp, X, codes, scales, torch.from_numpy(ref.mx4_values(code, byte)[:, :cols]), sp.SP_MX4_A16)


@pytest.mark.parametrize("T", [8, 9, 140])
def test_scales_of_every_size_in_a_row(sp, T):
    rows, cols = 70, 2048
    g = np.random.RandomState(T)
    code = g.randint(0, 16, (rows, cols // 32, 32))
    byte = g.randint(60, 200, (rows, cols // 32))
    # activations of a size that makes every block's products alike, 0 where that leaves binary16
    want = 127 - byte[0].astype(float)
    size = torch.from_numpy(np.where(np.abs(want) <= 12, 2.0 ** np.clip(want, -12, 12), 0.0)).repeat_interleave(32)
    byte[:] = byte[0]
    X = (torch.randn(T, cols, generator=torch.Generator().manual_seed(1)).double() * size).half()
    codes, scales = (torch.from_numpy(a) for a in ref.mx4_pack(code, byte))
    _check_product(sp, X, codes, scales, torch.from_numpy(ref.mx4_values(code, byte)), sp.SP_MX4_A16)


@pytest.mark.parametrize("T", [8, 9, 140])
def test_values_that_are_not_finite(sp, T):
    rows, cols = 140, 1024
    code, byte, X = _far_apart(rows, cols, T, 3)
    byte[5, 7], byte[13, 2] = 255, 255                               # NaN blocks, in a wide row too
    code[byte == 255] = 0
    X[1, 40], X[2, 70], X[3, 3] = float("inf"), float("nan"), float("-inf")   # 3: beside a large weight
    codes, scales = (torch.from_numpy(a) for a in ref.mx4_pack(code, byte))
    V = torch.from_numpy(ref.mx4_values(code, byte))
    Y = sp.sp_mx4_linear(X.cuda(), codes.cuda(), scales.cuda()).cpu().double()
    want = X.double() @ V.t()
    assert torch.equal(Y.isnan(), want.isnan())
    assert torch.equal(Y.isinf(), want.isinf()) and torch.equal(Y[want.isinf()], want[want.isinf()])
    fin = want.isfinite()
    bound = _product_bound(X.double().nan_to_num(0, 0, 0), V.nan_to_num(), torch.float16)
    assert ((Y - want).abs()[fin] <= bound[fin]).all()
