"""Products with 4-bit weights as a program calls them: without a workspace, captured in a graph, from
several threads."""
import threading

import pytest
import torch

from . import serve_reference as ref

pytestmark = pytest.mark.gpu

SIZES = [(0, 1), (0, 8), (0, 9), (0, 200), (1, 8), (1, 200)]      # mode, tokens


@pytest.fixture(scope="module")
def sp():
    from paper_2501_16376_b200 import binding
    yield binding
    assert binding.sp_wait_status() == 0


def _inputs(rows, cols, T, dtype, seed=0):
    codes, scales, _ = ref.mx4_random(rows, cols, seed, dtype=dtype)
    X = torch.randn(T, cols, generator=torch.Generator().manual_seed(seed)).to(dtype)
    return X.cuda(), codes.cuda(), scales.cuda()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("mode,T", SIZES)
def test_captured_calls_leave_the_same_bits(sp, mode, T, dtype):
    X, codes, scales = _inputs(300, 1037, T, dtype)
    want = sp.sp_mx4_linear(X, codes, scales, mode)
    fresh = torch.randn_like(X)
    want_fresh = sp.sp_mx4_linear(fresh, codes, scales, mode)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y = sp.sp_mx4_linear(X, codes, scales, mode)
        again = sp.sp_mx4_quantize(X)
        back = sp.sp_mx4_dequantize(*again, X.shape[1], dtype)
    for _ in range(2):
        graph.replay()
    assert torch.equal(Y, want)
    X.copy_(fresh)
    graph.replay()
    assert torch.equal(Y, want_fresh)
    assert torch.equal(back, sp.sp_mx4_dequantize(*sp.sp_mx4_quantize(fresh), X.shape[1], dtype))


def test_two_threads_on_their_own_streams(sp):
    cases = [(_inputs(500 + 64 * i, 2048, T, torch.bfloat16, i), mode) for i, (mode, T) in enumerate(SIZES)]
    want = [sp.sp_mx4_linear(*a, mode) for a, mode in cases]
    torch.cuda.synchronize()
    failures = []

    def work(which):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for i in range(60):
                    k = (i * (which + 1)) % len(cases)
                    a, mode = cases[k]
                    if not torch.equal(sp.sp_mx4_linear(*a, mode), want[k]):
                        failures.append((which, i))
        except Exception as e:                          # noqa: BLE001 - reported below
            failures.append(repr(e))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures
