"""A pruned transformer block served from 4-bit weights and an 8-bit key/value cache.

    python -m paper_2501_16376_b200.serve_block --workload llama3-8b --seqs 8 --prompt 256 --steps 32 --budget 128

The block's layers have the shapes of a workload of ``synth`` and random weights.  They are pruned
from calibration statistics (the workload's own rule: N:M groups or the running threshold),
quantised to microscaled 4-bit floats with the keep mask applied on the way, and the dense
matrices are dropped.  Prompts are taken in chunks (both operands of every product in 4 bits),
then tokens are generated one at a time (activations in 16 bits); the cache accumulates the
attention every token receives and, whenever it is full, keeps the ``--budget`` tokens that
received most.  One JSON line reports sizes and times.

Only the calls of the library do work that depends on the weights or the cache; normalisation,
gating and residuals are elementwise tensor operations.
"""
from __future__ import annotations

import argparse
import json

import torch

from . import binding as sp
from . import synth

#: head size by model width (64 for any other)
HEAD_DIM = {1024: 64, 4096: 128, 5120: 128}


class PackedLinear:
    """A pruned matrix in 4 bits."""

    def __init__(self, W: torch.Tensor, mask: torch.Tensor | None):
        self.rows, self.cols = W.shape
        self.codes, self.scales = sp.sp_mx4_quantize(W, mask)

    def __call__(self, x: torch.Tensor, mode: int) -> torch.Tensor:
        return sp.sp_mx4_linear(x, self.codes, self.scales, mode)

    def nbytes(self) -> int:
        return self.codes.numel() + self.scales.numel()


def _norm(x: torch.Tensor) -> torch.Tensor:
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-5)).to(x.dtype)


class ServedBlock:
    """One block: attention with grouped heads and a gated MLP, each after a normalisation and
    with a residual.  Generates for n_seqs sequences of equal length."""

    def __init__(self, w: synth.Workload, n_seqs: int, capacity: int, budget: int, recent: int,
                 block_tokens: int = 32, sparsity: float = 0.5, device="cuda"):
        layers = {layer.name: layer for layer in w.layers}
        self.width = layers["q_proj"].d_in
        self.head_dim = HEAD_DIM.get(self.width, 64)
        self.heads = layers["q_proj"].d_out // self.head_dim
        self.kv_heads = layers["k_proj"].d_out // self.head_dim
        self.n_seqs, self.budget, self.recent, self.capacity = n_seqs, budget, recent, capacity
        self.linear, self.dense_bytes = {}, 0
        for name, layer in layers.items():
            W = synth.gen_weight(w, 0, layer, device)
            X = synth.gen_activations(w, 0, layer.input, layer.d_in, 0, 1, device)
            with sp.Context(layer.d_in) as ctx:
                ctx.sp_calib_accumulate(X)
                if w.mode == "nm":
                    mask, _ = ctx.sp_select_nm(W, *w.patterns[0])
                else:
                    mask, _ = ctx.sp_select_unstructured(W, sparsity)
                self.linear[name] = PackedLinear(W, mask)
            self.dense_bytes += W.numel() * 2
        make = lambda tokens: sp.KvCache.empty(n_seqs, tokens, self.kv_heads, self.head_dim, block_tokens)
        self.cache, self.spare = make(capacity), make(capacity)
        self.acc = [torch.zeros(n_seqs, self.kv_heads, capacity, device=device) for _ in range(2)]
        self.length, self.evictions = 0, 0
        self.dtype = w.torch_dtype

    def _room(self, n: int):
        """Evicts down to the budget if n more tokens do not fit."""
        if self.length + n <= self.capacity:
            return
        if min(self.length, self.budget) + n > self.capacity:
            raise ValueError("%d tokens do not fit beside the %d kept of a cache of %d"
                             % (n, min(self.length, self.budget), self.capacity))
        lens = torch.full((self.n_seqs,), self.length, dtype=torch.int32, device="cuda")
        _, _, kept = self.cache.sp_cache_evict(lens, self.length, self.acc[0], self.budget, self.recent,
                                               self.spare, acc_out=self.acc[1])
        self.cache, self.spare = self.spare, self.cache
        self.acc.reverse()
        self.length = min(self.length, self.budget)
        self.evictions += 1

    def __call__(self, x: torch.Tensor, mode: int) -> torch.Tensor:
        """x [n_seqs, n, width] -> the block's output, the same shape; the n tokens join the cache."""
        B, n, _ = x.shape
        self._room(n)
        flat = lambda t: t.reshape(B * n, -1)
        h = flat(_norm(x))
        q = self.linear["q_proj"](h, mode).view(B, n, self.heads, self.head_dim)
        k = self.linear["k_proj"](h, mode).view(B, n, self.kv_heads, self.head_dim)
        v = self.linear["v_proj"](h, mode).view(B, n, self.kv_heads, self.head_dim)
        start = torch.full((B,), self.length, dtype=torch.int32, device=x.device)
        self.cache.sp_cache_append(k, v, start)
        self.length += n
        # accumulated in place: the call's own tokens start from 0
        o = self.cache.sp_cache_attention(q, start + n, self.length, acc_in=self.acc[0], acc_out=self.acc[0])
        x = x + self.linear["o_proj"](flat(o), mode).view_as(x)
        h = flat(_norm(x))
        up = torch.nn.functional.silu(self.linear["gate_proj"](h, mode)) * self.linear["up_proj"](h, mode)
        return x + self.linear["down_proj"](up, mode).view_as(x)


def run(w: synth.Workload, n_seqs: int, prompt: int, steps: int, budget: int, chunk: int = 32,
        recent: int = 16, sparsity: float = 0.5):
    """Takes a prompt, generates steps tokens; returns (block, outputs of the steps, report)."""
    if min(n_seqs, prompt, steps, chunk) < 1 or budget < 0:
        raise ValueError("sequences, prompt, steps and chunk are at least 1, the budget at least 0")
    capacity = max(prompt, budget + chunk)
    block = ServedBlock(w, n_seqs, capacity, budget, min(recent, budget), sparsity=sparsity)
    g = torch.Generator(device="cuda").manual_seed(synth.tensor_seed(w.seed, w.name, "serve"))
    x = torch.randn(n_seqs, prompt, block.width, generator=g, device="cuda").to(w.torch_dtype)
    for at in range(0, prompt, chunk):
        y = block(x[:, at:at + chunk], sp.SP_MX4_A4)
    outs, token = [], y[:, -1:]
    times = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    for i in range(steps):
        if i == min(3, steps - 1):
            times[0].record()
        token = block(_norm(token), sp.SP_MX4_A16)
        outs.append(token)
    times[1].record()
    torch.cuda.synchronize()
    packed = sum(m.nbytes() for m in block.linear.values())
    report = {"workload": w.name, "n_seqs": n_seqs, "prompt": prompt, "steps": steps,
              "us_per_step": times[0].elapsed_time(times[1]) * 1e3 / max(1, steps - min(3, steps - 1)),
              "weight_bytes_dense": block.dense_bytes, "weight_bytes": packed,
              "cache_tokens": block.length, "evictions": block.evictions,
              "finite": bool(torch.isfinite(torch.cat(outs)).all())}
    return block, outs, report


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workload", default="llama3-8b", choices=[n for n, w in synth.WORKLOADS.items()
                                                               if {"q_proj", "gate_proj"} <= {l.name for l in w.layers}])
    ap.add_argument("--seqs", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=256)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--budget", type=int, default=128, help="tokens kept when the cache is full")
    ap.add_argument("--sparsity", type=float, default=0.5)
    a = ap.parse_args()
    print(json.dumps(run(synth.WORKLOADS[a.workload], a.seqs, a.prompt, a.steps, a.budget, sparsity=a.sparsity)[2]))


if __name__ == "__main__":
    main()
