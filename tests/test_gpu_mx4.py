"""Microscaled 4-bit weights against the format's definition in binary64."""
import numpy as np
import pytest
import torch

from . import serve_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = [torch.float16, torch.bfloat16]
UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # half the spacing at 1
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}  # half the smallest subnormal


@pytest.fixture(scope="module")
def sp():
    from paper_2501_16376_b200 import binding
    yield binding
    assert binding.sp_wait_status() == 0


def _matrix(rows, cols, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(rows, cols, generator=g)
    w *= torch.exp2(torch.randint(-20, 12, (rows, (cols + 31) // 32), generator=g).float()).repeat_interleave(32, 1)[:, :cols]
    w[torch.rand(rows, cols, generator=g) < 0.3] = 0
    return w.to(dtype)


def _check_quantized(codes, scales, W):
    code, byte = ref.mx4_quantize(W)
    want_codes, want_scales = ref.mx4_pack(code, byte)
    assert np.array_equal(codes.cpu().numpy()[:, :want_codes.shape[1]], want_codes)
    assert np.array_equal(scales.cpu().numpy()[:want_scales.size], want_scales)
    return torch.from_numpy(ref.mx4_values(code, byte)[:, :W.shape[1]])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 33), (33, 8), (129, 130), (70, 264), (128, 1024), (300, 520)])
def test_quantize_and_back(sp, rows, cols, dtype):
    W = _matrix(rows, cols, dtype, rows * 1000 + cols)
    codes, scales = sp.sp_mx4_quantize(W.cuda())
    values = _check_quantized(codes, scales, W)
    back = sp.sp_mx4_dequantize(codes, scales, cols, dtype)
    assert torch.equal(back.cpu().double(), values)       # a 16-bit matrix's values fit its type


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_applies_a_mask_to_strided_rows_and_leaves_the_rest(sp, dtype):
    rows, cols = 150, 203
    big = _matrix(rows, cols + 22, dtype, 5).cuda()
    W = big[:, 5:5 + cols]                                 # not 16-byte aligned
    keep = torch.rand(rows, cols, generator=torch.Generator().manual_seed(1)) < 0.5
    bits = np.zeros((rows, (cols + 31) // 32 * 32), dtype=np.uint32)
    bits[:, :cols] = keep.numpy()
    words = (bits.reshape(rows, -1, 32) << np.arange(32, dtype=np.uint32)).sum(-1).astype(np.uint32).view(np.int32)
    codes = torch.full((rows, 160), 77, dtype=torch.uint8, device="cuda")   # 112 bytes needed
    scales = torch.full((sp.sp_mx4_scale_bytes(rows, cols) + 64,), 99, dtype=torch.uint8, device="cuda")
    sp.sp_mx4_quantize(W, torch.from_numpy(words).cuda(), codes, scales)
    values = _check_quantized(codes, scales, torch.where(keep, W.cpu(), torch.zeros((), dtype=dtype)))   # pruned: +0
    assert (codes[:, 112:] == 77).all() and (scales[-64:] == 99).all()
    out = torch.full((rows, cols + 9), 3.0, dtype=dtype, device="cuda")
    sp.sp_mx4_dequantize(codes, scales, cols, W_out=out[:, 2:2 + cols])
    assert torch.equal(out[:, 2:2 + cols].cpu().double(), values)
    assert (out[:, :2] == 3).all() and (out[:, 2 + cols:] == 3).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_special_values_and_ties(sp, dtype):
    top = torch.finfo(dtype).max
    small = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -133
    W = torch.zeros(12, 96)
    W[0, :16] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, 7.9])
    W[1, 0], W[1, 33], W[1, 70] = float("nan"), float("inf"), 1.0
    W[2, 0], W[2, 1], W[2, 40] = top, -top, 1.0
    W[3, 0], W[3, 33], W[3, 34] = small, 3 * small, -small
    W[4, :32] = -0.0
    W[5, 0], W[5, 1] = 4.0, 1e-3
    W[6, :32] = torch.linspace(-8, 8, 32)
    W = W.to(dtype)
    codes, scales = sp.sp_mx4_quantize(W.cuda())
    values = _check_quantized(codes, scales, W)
    back = sp.sp_mx4_dequantize(codes, scales, 96, dtype).cpu().double()
    assert torch.equal(back.isnan(), values.isnan()) and torch.equal(back.nan_to_num(), values.nan_to_num())
    assert back[1, 70] == 1 and back[1, :64].isnan().all()


def _product_bound(X, V, dtype):
    """One rounding to the output type and one of binary32 for every addition, whatever the order."""
    mag = X.abs() @ V.abs().t()
    return (X @ V.t()).abs() * UNIT[dtype] + mag * (X.shape[1] + 32) * 2.0 ** -23 * 1.01 + TINY[dtype]


def _check_product(sp, X, codes, scales, V, mode):
    Y = sp.sp_mx4_linear(X.cuda(), codes.cuda(), scales.cuda(), mode).cpu().double()
    x = X.double()
    if mode == sp.SP_MX4_A4:
        x = torch.from_numpy(ref.mx4_values(*ref.mx4_quantize(X))[:, :X.shape[1]])
    want = x @ V.t()
    assert Y.shape == want.shape
    assert ((Y - want).abs() <= _product_bound(x, V, X.dtype)).all()


TOKENS = [1, 2, 7, 8, 9, 16, 17, 32, 33, 64, 65, 127, 128, 129, 200, 257, 300]


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(128, 256), (200, 640), (257, 1000), (96, 4096)])
def test_product(sp, rows, cols, dtype, mode):
    codes, scales, V = ref.mx4_random(rows, cols, rows + cols, dtype=dtype)
    g = torch.Generator().manual_seed(cols)
    for T in TOKENS:
        X = torch.randn(T, cols, generator=g)
        X[:, :: 97] *= 20
        _check_product(sp, X.to(dtype), codes, scales, V, mode)


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols,T", [(1, 1, 1), (1, 31, 3), (5, 33, 40), (1, 128, 300), (127, 95, 130), (130, 129, 20),
                                         (300, 2817, 5), (129, 33, 513)])
def test_product_of_odd_sizes(sp, rows, cols, T, dtype, mode):
    codes, scales, V = ref.mx4_random(rows, cols, rows * cols, dtype=dtype)
    X = torch.randn(T, cols, generator=torch.Generator().manual_seed(T)).to(dtype)
    _check_product(sp, X, codes, scales, V, mode)


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("rows,cols,T", [(10000, 130, 140), (15000, 96, 150), (20000, 96, 20), (25000, 96, 20), (30000, 96, 9),
                                         (40000, 130, 20), (40000, 96, 140), (40000, 96, 400), (20000, 1100, 40), (19000, 1100, 260)])
def test_product_of_many_rows(sp, rows, cols, T, mode):
    # tiles of every height, several of them for a block, in both tile kernels
    codes, scales, V = ref.mx4_random(rows, cols, rows + cols)
    X = torch.randn(T, cols, generator=torch.Generator().manual_seed(T)).to(torch.bfloat16 if T % 20 else torch.float16)
    _check_product(sp, X, codes, scales, V, mode)


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("T", [1, 12, 150])
def test_product_of_strided_tensors_on_another_stream(sp, T, mode):
    rows, cols, dtype = 200, 520, torch.bfloat16
    codes, scales, V = ref.mx4_random(rows, cols, 9)
    wide = torch.randn(T + 1, cols + 11, generator=torch.Generator().manual_seed(2)).to(dtype)
    stream = torch.cuda.Stream()
    big, pitched = wide.cuda(), torch.zeros(rows, 320, dtype=torch.uint8, device="cuda")
    pitched[:, :272] = codes.cuda()
    sc = scales.cuda()
    for off in (0, 3, 8):
        out = torch.full((T, rows + 7), 5.0, dtype=dtype, device="cuda")
        torch.cuda.synchronize()
        sp.sp_mx4_linear(big[1:, off:off + cols], pitched[:, :272], sc, mode, Y=out[:, 3:3 + rows], stream=stream)
        stream.synchronize()
        x = wide[1:, off:off + cols]
        xd = x.double() if mode == 0 else torch.from_numpy(ref.mx4_values(*ref.mx4_quantize(x))[:, :cols])
        err = (out[:, 3:3 + rows].cpu().double() - xd @ V.t()).abs()
        assert (err <= _product_bound(xd, V, dtype)).all()
        assert (out[:, :3] == 5).all() and (out[:, 3 + rows:] == 5).all()


@pytest.mark.parametrize("T", [1, 20, 140])
def test_product_of_bf16_activations_far_apart(sp, T):
    # beside elements up to 2^60 times larger that meet only pruned weights, small ones still count
    rows, cols = 70, 512
    codes, scales, V = ref.mx4_random(rows, cols, 4)
    code, byte = ref.mx4_quantize(torch.zeros(rows, cols))
    w = torch.randn(rows, cols, generator=torch.Generator().manual_seed(3)) * 0.02
    w[:, 5::32] = 0
    code, byte = ref.mx4_quantize(w)
    codes, scales = (torch.from_numpy(a) for a in ref.mx4_pack(code, byte))
    V = torch.from_numpy(ref.mx4_values(code, byte))
    X = torch.randn(T, cols, generator=torch.Generator().manual_seed(8))
    X[:, 5::32] *= 2.0 ** 60
    X = X.to(torch.bfloat16)
    _check_product(sp, X, codes, scales, V, sp.SP_MX4_A16)


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [3, 140])
def test_product_with_values_that_are_not_finite(sp, T, dtype, mode):
    rows, cols = 140, 256
    w = torch.randn(rows, cols, generator=torch.Generator().manual_seed(3)) * 0.02
    w[:, 64:96] = 0
    w[7, 40] = float("nan")
    code, byte = ref.mx4_quantize(w)
    codes, scales = (torch.from_numpy(a) for a in ref.mx4_pack(code, byte))
    X = torch.randn(T, cols, generator=torch.Generator().manual_seed(8)).to(dtype)
    X[1, 70] = float("inf")                                 # inf * 0: NaN for every row
    X[2, 3] = float("nan")
    Y = sp.sp_mx4_linear(X.cuda(), codes.cuda(), scales.cuda(), mode).cpu()
    bad = torch.zeros(T, rows, dtype=torch.bool)
    bad[:, 7] = True
    bad[1:3] = True
    assert torch.equal(~Y.isfinite(), bad)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [2, 140])
def test_product_over_the_whole_range_of_scales(sp, T, dtype):
    # every block of a row with a scale of its own, from 2^-127 to 2^40, weights of every code
    rows, cols = 40, 1024
    g = np.random.RandomState(0)
    code = g.randint(0, 16, (rows, 32, 32))
    byte = g.randint(60, 150, (rows, 32))
    byte[0], byte[1, ::2] = 0, 0
    codes, scales = (torch.from_numpy(a) for a in ref.mx4_pack(code, byte))
    V = torch.from_numpy(ref.mx4_values(code, byte))
    X = torch.randn(T, cols, generator=torch.Generator().manual_seed(8)).to(dtype)
    if dtype == torch.float16:
        byte = g.randint(120, 130, (rows, 32))
        codes, scales = (torch.from_numpy(a) for a in ref.mx4_pack(code, byte))
        V = torch.from_numpy(ref.mx4_values(code, byte))
    _check_product(sp, X, codes, scales, V, sp.SP_MX4_A16)


@pytest.mark.parametrize("mode", [0, 1])
def test_product_gives_the_same_bits_twice(sp, mode):
    codes, scales, V = ref.mx4_random(512, 2048, 4)
    codes, scales = codes.cuda(), scales.cuda()
    for T in (1, 30, 300):
        X = torch.randn(T, 2048, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
        first = sp.sp_mx4_linear(X, codes, scales, mode).clone()
        for _ in range(3):
            assert torch.equal(sp.sp_mx4_linear(X, codes, scales, mode), first)


def test_empty_matrices_are_fine(sp):
    codes, scales, V = ref.mx4_random(64, 64, 4)
    Y = sp.sp_mx4_linear(torch.zeros(0, 64, dtype=torch.float16, device="cuda"), codes.cuda(), scales.cuda())
    assert Y.shape == (0, 64)
    c, s = sp.sp_mx4_quantize(torch.zeros(0, 64, dtype=torch.float16, device="cuda"))
    assert c.shape == (0, 32) and s.numel() == 0


def test_binding_refusals(sp):
    codes, scales, V = ref.mx4_random(64, 64, 4)
    X = torch.zeros(2, 64, dtype=torch.float16, device="cuda")
    cc, cs = codes.cuda(), scales.cuda()
    for bad in (lambda: sp.sp_mx4_linear(X.float(), cc, cs), lambda: sp.sp_mx4_linear(X.cpu(), cc, cs),
                lambda: sp.sp_mx4_linear(X, cc[:, :16], cs), lambda: sp.sp_mx4_linear(X, cc, cs[:100]),
                lambda: sp.sp_mx4_linear(X, cc, cs, 7), lambda: sp.sp_mx4_linear(X, codes, scales),
                lambda: sp.sp_mx4_linear(X, cc, cs, Y=torch.zeros(2, 63, dtype=X.dtype, device="cuda")),
                lambda: sp.sp_mx4_linear(X, cc, cs, Y=torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")),
                lambda: sp.sp_mx4_quantize(X, mask=torch.zeros(2, 1, dtype=torch.int32, device="cuda")),
                lambda: sp.sp_mx4_quantize(X, codes=cc[1:3, 1:33]),
                lambda: sp.sp_mx4_dequantize(cc, cs, 64, W_out=torch.zeros(64, 65, dtype=X.dtype, device="cuda"))):
        with pytest.raises(sp.SpError):
            bad()
