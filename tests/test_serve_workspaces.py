"""Which products with 4-bit weights take scratch memory (no GPU needed: the library's entry points are
replaced, and CPU tensors stand for those of the device)."""
import pytest
import torch


@pytest.fixture
def sp(monkeypatch):
    from paper_2501_16376_b200 import binding
    real, calls = binding.lib, []

    class Library:
        def __getattr__(self, name):
            if name != "sp_mx4_linear":
                return getattr(real, name)
            return lambda *a: calls.append((a[12], a[13])) or binding.SP_OK
    monkeypatch.setattr(binding, "lib", Library())
    monkeypatch.setattr(binding, "_current_device", lambda: -1)
    monkeypatch.setattr(binding, "_raw_stream", lambda stream, device: 0)
    monkeypatch.setattr(binding, "calls", calls, raising=False)
    return binding


@pytest.mark.parametrize("mode,tokens,offset,pitch,needed", [
    (0, 4, 0, 64, False), (0, 4, 1, 67, False), (1, 4, 0, 64, False),          # few tokens: none
    (0, 300, 0, 64, False), (0, 300, 8, 72, False),                            # rows on 16-byte boundaries
    (0, 300, 1, 72, True), (0, 300, 0, 67, True),                              # rows that are not
    (1, 300, 0, 64, True)])                                                    # the quantised activations
def test_scratch_memory_is_asked_for_where_it_is_used(sp, mode, tokens, offset, pitch, needed):
    X = torch.zeros(tokens * pitch + 16, dtype=torch.float16)[offset:].as_strided((tokens, 64), (pitch, 1))
    Y = torch.zeros(tokens, 32, dtype=torch.float16)
    codes, scales = torch.zeros(32, 32, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8)
    sp.sp_mx4_linear(X, codes, scales, mode, Y=Y)
    pointer, size = sp.calls[-1]
    if needed:
        assert pointer and size == sp.sp_mx4_linear_workspace(tokens, 32, 64, mode) > 0
    else:
        assert pointer is None and size == 0
