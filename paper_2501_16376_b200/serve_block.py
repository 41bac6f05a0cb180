"""A pruned transformer block served from 4-bit weights and an 8-bit key/value cache.

    python -m paper_2501_16376_b200.serve_block --workload llama3-8b --seqs 8 --prompt 256 --steps 32 --budget 128

The block's layers have the shapes of a workload of ``synth`` and random weights.  They are pruned
from calibration statistics (the workload's own rule: N:M groups or the running threshold),
quantised to microscaled 4-bit floats with the keep mask applied on the way, and the dense
matrices are dropped.  Prompts are taken in chunks (both operands of every product in 4 bits),
then tokens are generated one at a time (activations in 16 bits); the cache accumulates the
attention every token receives and, whenever it is full, keeps the ``--budget`` tokens that
received most.  One JSON line reports sizes and times.

    python -m paper_2501_16376_b200.serve_block --workload llama3-8b --seqs 4 --answers 8 --prompt 1024 --steps 64

With ``--answers`` every prompt is answered several times: queries and keys carry their positions, the
prompt's blocks are shared by its answers (a table row forked for each, own copies of the last block),
and the attention over a prompt is computed once for all its answers.

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
        self._prune(w, sparsity, device)
        self.n_seqs, self.budget, self.recent, self.capacity = n_seqs, budget, recent, capacity
        make = lambda tokens: sp.KvCache.empty(n_seqs, tokens, self.kv_heads, self.head_dim, block_tokens)
        self.cache, self.spare = make(capacity), make(capacity)
        self.acc = [torch.zeros(n_seqs, self.kv_heads, capacity, device=device) for _ in range(2)]
        self.length, self.evictions = 0, 0

    def _prune(self, w: synth.Workload, sparsity: float, device):
        """The layers, pruned and in 4 bits; the sizes of heads."""
        layers = {layer.name: layer for layer in w.layers}
        self.width = layers["q_proj"].d_in
        self.head_dim = HEAD_DIM.get(self.width, 64)
        self.heads = layers["q_proj"].d_out // self.head_dim
        self.kv_heads = layers["k_proj"].d_out // self.head_dim
        self.linear, self.dense_bytes = {}, 0
        self.dtype = w.torch_dtype
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
        q, k, v = self._project(x, mode)
        start = torch.full((B,), self.length, dtype=torch.int32, device=x.device)
        self.cache.sp_cache_append(k, v, start)
        self.length += n
        # accumulated in place: the call's own tokens start from 0
        o = self.cache.sp_cache_attention(q, start + n, self.length, acc_in=self.acc[0], acc_out=self.acc[0])
        return self._rest(x, o, mode)

    def _project(self, x: torch.Tensor, mode: int):
        B, n, _ = x.shape
        h = _norm(x).reshape(B * n, -1)
        return (self.linear[name](h, mode).view(B, n, heads, self.head_dim)
                for name, heads in (("q_proj", self.heads), ("k_proj", self.kv_heads), ("v_proj", self.kv_heads)))

    def _rest(self, x: torch.Tensor, o: torch.Tensor, mode: int) -> torch.Tensor:
        """The block after its attention."""
        flat = lambda t: t.reshape(x.shape[0] * x.shape[1], -1)
        x = x + self.linear["o_proj"](flat(o), mode).view_as(x)
        h = flat(_norm(x))
        up = torch.nn.functional.silu(self.linear["gate_proj"](h, mode)) * self.linear["up_proj"](h, mode)
        return x + self.linear["down_proj"](up, mode).view_as(x)


class AnsweringBlock(ServedBlock):
    """One block that answers n_prompts prompts of equal length, each `answers` times.  Sequence
    p * answers + i is the i-th answer of prompt p; the prompt is taken on the first one's row of the
    table.  Positions are rotated with base theta; qk_norm normalises the heads of queries and keys."""

    def __init__(self, w: synth.Workload, n_prompts: int, answers: int, prompt: int, new: int,
                 block_tokens: int = 32, theta: float = 10000.0, qk_norm: bool = False,
                 sparsity: float = 0.5, device="cuda"):
        self._prune(w, sparsity, device)
        self.n_prompts, self.answers, self.n_seqs, self.prompt = n_prompts, answers, n_prompts * answers, prompt
        per = lambda tokens: (tokens + block_tokens - 1) // block_tokens
        # a prompt's blocks once, and for every answer its new ones and a copy of the prompt's last
        blocks = n_prompts * per(prompt) + self.n_seqs * (per(prompt % block_tokens + new))
        c = self.cache = sp.KvCache.pool(self.n_seqs, prompt + new, blocks, self.kv_heads, self.head_dim, block_tokens, device)
        self.prompts = sp.KvCache(c.k, c.v, c.k_scale, c.v_scale, c.table[::answers], refs=c.refs)
        i32 = dict(dtype=torch.int32, device=device)
        self.group_start = torch.arange(0, self.n_seqs + 1, answers, **i32)
        self.prefix = torch.full((n_prompts,), prompt, **i32)
        rows = torch.arange(self.n_seqs, **i32).view(n_prompts, answers)
        self.first, self.others = rows[:, :1].flatten(), rows[:, 1:].flatten()
        self.freq = (theta ** (-torch.arange(0, self.head_dim, 2, dtype=torch.float64, device=device) / self.head_dim)).float()
        self.head_norm = torch.ones(self.head_dim, dtype=self.dtype, device=device) if qk_norm else None
        self.missing = torch.zeros(1, **i32)               # blocks that a call asked for in vain
        self.length, self.forked = 0, False

    def fork(self):
        """The prompts have been taken: their answers begin, from the same blocks."""
        self.cache.sp_cache_fork(self.others, self.first.repeat_interleave(self.answers - 1))
        self.forked = True

    def end(self) -> int:
        """Gives back all answers but each prompt's first; returns the blocks in use, at the front of
        the pool."""
        self.cache.sp_cache_fork(self.others)
        self.forked = False
        return int(self.cache.sp_cache_compact())

    def __call__(self, x: torch.Tensor, mode: int) -> torch.Tensor:
        """x [n_prompts (after fork: n_prompts * answers), n, width] -> the block's output."""
        B, n, _ = x.shape
        cache = self.cache if self.forked else self.prompts
        if self.length + n > cache.table.shape[1] * cache.block_tokens:
            raise ValueError("%d tokens do not fit behind %d" % (n, self.length))
        start = torch.full((B,), self.length, dtype=torch.int32, device=x.device)
        self.missing += cache.sp_cache_reserve(start, n)[:1]
        q, k, v = self._project(x, mode)
        q, k = sp.sp_qk_norm_rotary(q, k, start, self.freq, self.head_norm, self.head_norm, Q_out=q, K_out=k)
        cache.sp_cache_append(k, v, start)
        self.length += n
        if self.forked:
            o = cache.sp_cache_attention_shared(q, start + n, self.length, self.group_start, self.prefix, self.prompt, self.answers)
        else:
            o = cache.sp_cache_attention(q, start + n, self.length)
        return self._rest(x, o, mode)


def run_answers(w: synth.Workload, n_prompts: int, answers: int, prompt: int, steps: int, chunk: int = 32,
                theta: float = 10000.0, qk_norm: bool = False, sparsity: float = 0.5, first=None):
    """Takes n_prompts prompts, answers each several times for steps tokens; first: the answers' first
    tokens [n_prompts * answers, 1, width] (default: random).  Returns (block, outputs of the steps, report)."""
    if min(n_prompts, answers, prompt, steps, chunk) < 1:
        raise ValueError("prompts, answers, tokens of a prompt, steps and chunk are at least 1")
    block = AnsweringBlock(w, n_prompts, answers, prompt, steps, theta=theta, qk_norm=qk_norm, sparsity=sparsity)
    g = torch.Generator(device="cuda").manual_seed(synth.tensor_seed(w.seed, w.name, "answers"))
    x = torch.randn(n_prompts, prompt, block.width, generator=g, device="cuda").to(w.torch_dtype)
    for at in range(0, prompt, chunk):
        block(x[:, at:at + chunk], sp.SP_MX4_A4)
    block.fork()
    if first is None:
        first = torch.randn(block.n_seqs, 1, block.width, generator=g, device="cuda").to(w.torch_dtype)
    outs, token, warm = [], first, min(3, steps - 1)
    times = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    for i in range(steps):
        if i == warm:
            times[0].record()
        token = block(_norm(token), sp.SP_MX4_A16)
        outs.append(token)
    times[1].record()
    torch.cuda.synchronize()
    used = int((block.cache.refs > 0).sum())
    report = {"workload": w.name, "prompts": n_prompts, "answers": answers, "prompt": prompt, "steps": steps,
              "us_per_step": times[0].elapsed_time(times[1]) * 1e3 / (steps - warm),
              "cache_blocks": used, "cache_blocks_missing": int(block.missing), "cache_blocks_after": block.end(),
              "cache_blocks_unshared": block.n_seqs * -(-block.length // block.cache.block_tokens),
              "finite": bool(torch.isfinite(torch.cat(outs)).all())}
    return block, outs, report


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
    ap.add_argument("--answers", type=int, default=0, help="answers of every one of --seqs prompts (0: one, with eviction)")
    ap.add_argument("--theta", type=float, default=10000.0, help="base of the rotated positions, with --answers")
    ap.add_argument("--qk-norm", action="store_true", help="normalise the heads of queries and keys, with --answers")
    a = ap.parse_args()
    if a.answers:
        print(json.dumps(run_answers(synth.WORKLOADS[a.workload], a.seqs, a.answers, a.prompt, a.steps, theta=a.theta,
                                     qk_norm=a.qk_norm, sparsity=a.sparsity)[2]))
        return
    print(json.dumps(run(synth.WORKLOADS[a.workload], a.seqs, a.prompt, a.steps, a.budget, sparsity=a.sparsity)[2]))


if __name__ == "__main__":
    main()
