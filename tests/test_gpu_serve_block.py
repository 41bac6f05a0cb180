"""The serving example: a pruned block from 4-bit weights and an 8-bit cache, against the same
block computed from the stored values in binary64."""
import math

import numpy as np
import pytest
import torch

from . import serve_reference as ref

pytestmark = pytest.mark.gpu


def _values(linear):
    from paper_2501_16376_b200 import binding as sp
    nb = (linear.cols + 31) // 32
    c = linear.codes.cpu().numpy().astype(int)[:, :nb * 16]
    code = np.stack([c & 15, c >> 4], -1).reshape(linear.rows, nb, 32)
    kt = (nb + 3) // 4
    r, b = np.arange(linear.rows)[:, None], np.arange(nb)[None]
    byte = linear.scales.cpu().numpy().astype(int)[(r // 128 * kt + b // 4) * 512 + r % 32 * 16 + r // 32 % 4 * 4 + b % 4]
    return torch.from_numpy(ref.mx4_values(code, byte)[:, :linear.cols])


def _norm(x, dtype):
    f = x.double()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-5)).to(dtype).double()


@pytest.mark.parametrize("workload", ["llama3-8b", "llama2-7b"])
def test_a_block_is_served_from_what_it_stored(workload):
    from paper_2501_16376_b200 import binding as sp
    from paper_2501_16376_b200 import serve_block, synth
    w = synth.scaled(synth.WORKLOADS[workload], blocks=1, n_seqs=1, seq_len=64, shrink=8)
    block, outs, report = serve_block.run(w, n_seqs=2, prompt=40, steps=20, budget=24, chunk=16, recent=4)
    assert report["evictions"] >= 1 and report["finite"]
    assert report["weight_bytes"] < 0.28 * report["weight_bytes_dense"]
    assert block.length <= block.capacity and len(outs) == 20
    # accumulated weights of the cached tokens: every query has handed out 1 per head of a group
    assert (block.acc[0][..., :block.length] >= 0).all()

    # one more token, recomputed from the stored weights and cache in binary64 (rounded where the
    # block rounds: after each product, the attention, the gate and each sum)
    dt = block.dtype
    x = torch.randn(2, 1, block.width, generator=torch.Generator().manual_seed(5)).to(dt)
    block._room(1)
    W = {n: _values(m) for n, m in block.linear.items()}
    lin = lambda n, t: (t.double() @ W[n].t()).to(dt)
    h = _norm(x, dt).reshape(2, -1)
    q, k, v = (lin(n, h) for n in ("q_proj", "k_proj", "v_proj"))
    before = ref.PlainCache(block.cache)
    start = [block.length] * 2
    before.append(k.view(2, 1, block.kv_heads, -1), v.view(2, 1, block.kv_heads, -1), start)
    y = block(x.cuda(), sp.SP_MX4_A16).cpu()
    o = before.attention(q.view(2, 1, block.heads, -1), [s + 1 for s in start], block.length, block.head_dim ** -0.5)[0]
    o = torch.from_numpy(o).to(dt).reshape(2, -1)
    a = (x.reshape(2, -1).double() + lin("o_proj", o).double()).to(dt)
    h = _norm(a, dt)
    gate = lin("gate_proj", h)
    up = (torch.nn.functional.silu(gate.double()).to(dt).double() * lin("up_proj", h).double()).to(dt)
    want = (a.double() + lin("down_proj", up).double()).to(dt).double()
    got = y.reshape(2, -1).double()
    # a dozen roundings to 16 bits in a chain, each at most one unit relative to its operands
    unit = 2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -11
    assert ((got - want).norm() / want.norm()).item() <= 12 * unit
    assert math.isfinite(got.norm().item())


def test_the_command_prints_one_json_line(capsys, monkeypatch):
    import json
    import sys

    from paper_2501_16376_b200 import serve_block
    monkeypatch.setattr(sys, "argv", ["serve_block", "--workload", "llama3-8b", "--seqs", "2", "--prompt", "64",
                                      "--steps", "4", "--budget", "32"])
    serve_block.main()
    out = json.loads(capsys.readouterr().out)
    assert out["finite"] and out["cache_tokens"] > 0 and out["us_per_step"] > 0
