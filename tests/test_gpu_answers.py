"""The serving example that answers a prompt several times: positions, shared blocks and the attention
over a shared prompt together, against the same block without sharing."""
import json
import sys

import pytest
import torch

from . import answers_reference as answers
from . import serve_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sb():
    from paper_2501_16376_b200 import serve_block
    return serve_block


def _workload(name):
    from paper_2501_16376_b200 import synth
    return synth.scaled(synth.WORKLOADS[name], blocks=1, n_seqs=1, seq_len=64, shrink=8)


@pytest.mark.parametrize("workload,qk_norm", [("llama3-8b", True), ("llama2-7b", False)])
@pytest.mark.parametrize("prompt", [70, 96])
def test_answers_are_those_of_each_alone(sb, workload, qk_norm, prompt):
    """Prompts that end inside a block and at its end; each answer is also computed alone.  Only the
    attention's order of sums differs: 2^-9 (bf16) of the outputs is one rounding, and what a step
    starts from differs by those of the steps before."""
    w = _workload(workload)
    g = torch.Generator().manual_seed(3)
    first = torch.randn(6, 1, 512, generator=g).to(w.torch_dtype).cuda()
    block, outs, report = sb.run_answers(w, 2, 3, prompt, 5, qk_norm=qk_norm, first=first)
    assert report["finite"] and report["cache_blocks_missing"] == 0
    assert report["cache_blocks_after"] <= report["cache_blocks"] < report["cache_blocks_unshared"]
    refs = block.cache.refs.tolist()
    assert all(r > 0 for r in refs[:report["cache_blocks_after"]]) and not any(refs[report["cache_blocks_after"]:])
    for i in range(3):
        _, alone, _ = sb.run_answers(w, 2, 1, prompt, 5, qk_norm=qk_norm, first=first[i::3])
        for step, (a, b) in enumerate(zip(outs, alone)):
            a, b = a[i::3].double(), b.double()
            unit = torch.finfo(w.torch_dtype).eps / 2
            assert ((a - b).norm() / b.norm()).item() <= 4 * (step + 1) * unit


def test_a_step_against_its_parts(sb):
    """One step of the answers: the keys that are in the cache, and the attention, from the definitions."""
    from paper_2501_16376_b200 import binding as sp
    w = _workload("llama3-8b")
    block, _, _ = sb.run_answers(w, 1, 1, 40, 1)
    block = sb.AnsweringBlock(w, 2, 3, 50, 4, qk_norm=True)
    x = torch.randn(2, 50, block.width, generator=torch.Generator().manual_seed(1)).to(w.torch_dtype).cuda()
    block(x, sp.SP_MX4_A4)
    block.fork()
    y = torch.randn(6, 1, block.width, generator=torch.Generator().manual_seed(2)).to(w.torch_dtype).cuda()
    q, k, v = block._project(y, sp.SP_MX4_A16)
    start = torch.full((6,), 50, dtype=torch.int32, device="cuda")
    pages = answers.PlainPages(block.cache)
    assert tuple(block.cache.sp_cache_reserve(start, 1).tolist()) == pages.reserve([50] * 6, 1)
    pages.check(block.cache)
    q2, k2 = sp.sp_qk_norm_rotary(q, k, start, block.freq, block.head_norm, block.head_norm)
    want, mag = answers.norm_rotary(k, block.head_norm, [50] * 6, block.freq, False, 1e-6)
    assert (abs(k2.double().cpu().numpy() - want) <= torch.finfo(w.torch_dtype).eps / 2 * abs(want) + 2.0 ** -19 * mag).all()
    block.cache.sp_cache_append(k2, v, start)
    plain = ref.PlainCache(block.cache)
    O, _, _, m, terms = plain.attention(q2, [51] * 6, 51, block.head_dim ** -0.5)
    got = block.cache.sp_cache_attention_shared(q2, start + 1, 51, block.group_start, block.prefix, 50, 3).double().cpu().numpy()
    d = (block.head_dim / 16 + 4) * 2.0 ** -22 * terms[..., None]
    assert (abs(got - O) <= torch.finfo(w.torch_dtype).eps / 2 * abs(O) + (4 * d + 2.0 ** -17 + 2.0 ** -20) * m).all()


def test_more_tokens_than_there_is_room_for(sb):
    from paper_2501_16376_b200 import binding as sp
    block = sb.AnsweringBlock(_workload("llama3-8b"), 1, 2, 32, 1)
    x = torch.zeros(1, 65, block.width, dtype=block.dtype, device="cuda")
    with pytest.raises(ValueError):
        block(x, sp.SP_MX4_A4)
    assert block.length == 0


def test_the_command(sb, capsys, monkeypatch):
    monkeypatch.setattr(sys, "argv", ["serve_block", "--workload", "llama3-8b", "--seqs", "2", "--answers", "4", "--prompt", "100",
                                      "--steps", "4", "--qk-norm"])
    sb.main()
    out = json.loads(capsys.readouterr().out)
    assert out["finite"] and out["cache_blocks_missing"] == 0 and out["us_per_step"] > 0
