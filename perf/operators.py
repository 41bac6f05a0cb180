"""Measured cases of the operators that serve a pruned model: microscaled 4-bit weights (their
quantisation and their product) and the 8-bit key/value cache (append, attention, eviction).

Sizes are those of the layer shapes the package prunes (LLaMA-2-7B, LLaMA-3-8B, LLaMA-2-13B and
Pythia-410M: widths 1024 / 4096 / 5120, feed-forward 4096 / 11008 / 13824 / 14336, head sizes 64
and 128, 8 to 40 heads) and ragged ones beside them.

``run`` computes an operator from elementary torch operations in binary32, or, with ``own`` set,
calls the library.  Data layouts (both forms read and write the same):

  codes   uint8 [rows, pitch]: two 4-bit codes a byte, the even column in the low half; a row's
          blocks of 32 columns take 16 bytes each; the pitch is a multiple of 16 bytes.
  scales  uint8, tiles of 512 bytes for 128 rows x 4 blocks: byte (r % 32) * 16 + (r / 32) * 4 + b
          of a tile is the scale of row r, block b; tiles run along a row of tiles first.
  cache   e4m3 codes [blocks, kv heads, tokens of a block, head size] and binary32 scales
          [blocks, kv heads], for K and for V; a table [sequences, blocks] names the blocks.
"""
import math

import torch

own = False

DEV = "cuda"
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)      # magnitudes of the 4-bit code
MOST_LINEAR = 8191 * 4096 * 14336                    # multiply-adds of the largest listed product
MOST_QUANT = 14336 * 4096
MOST_CACHE = 32 * 8191 * 8                           # (token, kv head) pairs of the largest cache


def listed():
    return [
        # a small layer: the call is all launch and latency
        dict(name="quantize 512x512 masked f16", op="quantize", rows=512, cols=512, dtype="f16", masked=True),
        # the largest matrix of a LLaMA-3-8B block, 2:4-pruned beforehand
        dict(name="quantize 14336x4096 bf16", op="quantize", rows=14336, cols=4096, dtype="bf16", masked=False),
        # one token through an attention projection: a decoding step
        dict(name="linear a16 1x4096x4096 bf16", op="linear", mode="a16", tokens=1, cols=4096, rows=4096, dtype="bf16"),
        # a ragged batch of prompts kept at 16-bit activations, LLaMA-2-7B's feed-forward
        dict(name="linear a16 333x4096x11008 f16", op="linear", mode="a16", tokens=333, cols=4096, rows=11008, dtype="f16"),
        # a prompt of medium length, LLaMA-2-13B's down projection, both sides in 4 bits
        dict(name="linear a4 512x13824x5120 bf16", op="linear", mode="a4", tokens=512, cols=13824, rows=5120, dtype="bf16"),
        # the longest prompt batch, one token short of a round number
        dict(name="linear a4 8191x4096x14336 bf16", op="linear", mode="a4", tokens=8191, cols=4096, rows=14336, dtype="bf16"),
        # one new token for each of 64 sequences (LLaMA-3-8B's 8 kv heads)
        dict(name="append 64x1 bf16", op="append", seqs=64, new=1, before=700, kv_heads=8, head=128, block=32, dtype="bf16"),
        # prompts of odd length, LLaMA-2-7B's 32 kv heads
        dict(name="append 4x2047 f16", op="append", seqs=4, new=2047, before=0, kv_heads=32, head=128, block=64, dtype="f16"),
        # a short conversation of Pythia-410M, four speculated tokens at once
        dict(name="attention 1x517 q4 f16", op="attention", seqs=1, length=517, queries=4, kv_heads=16, group=1, head=64, block=16, weights=False, dtype="f16"),
        # a full decoding batch of LLaMA-3-8B, accumulating the weights that eviction needs
        dict(name="attention 32x8191 bf16", op="attention", seqs=32, length=8191, queries=1, kv_heads=8, group=4, head=128, block=32, weights=True, dtype="bf16"),
        # one conversation back to a quarter
        dict(name="evict 1x1001 to 256", op="evict", seqs=1, length=1001, budget=256, recent=32, kv_heads=8, head=128, block=32),
        # long documents back to an eighth
        dict(name="evict 8x32768 to 4096", op="evict", seqs=8, length=32768, budget=4096, recent=128, kv_heads=8, head=128, block=32),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "append", "attention", "attention", "evict"])
    dtype = rng.choice(["f16", "bf16"])
    if op == "quantize":
        rows, cols = _log(rng, 64, 16384), _log(rng, 64, 14336)
        rows = max(1, min(rows, MOST_QUANT // cols))
        return dict(op=op, rows=rows, cols=cols, dtype=dtype, masked=rng.random() < 0.5)
    if op == "linear":
        cols, rows = _log(rng, 256, 14336), _log(rng, 256, 14336)
        if rng.random() < 0.7:                       # most layers are multiples of 128 wide
            cols, rows = max(256, cols // 128 * 128), max(256, rows // 128 * 128)
        tokens = max(1, min(_log(rng, 1, 8192), MOST_LINEAR // (rows * cols)))
        return dict(op=op, mode=rng.choice(["a16", "a4"]), tokens=tokens, cols=cols, rows=rows, dtype=dtype)
    kv_heads, head, block = rng.choice([1, 2, 5, 8, 16, 32]), rng.choice([64, 128]), rng.choice([16, 32, 64])
    if op == "append":
        seqs, new = _log(rng, 1, 64), _log(rng, 1, 2048)
        new = max(1, min(new, 8192 // seqs))
        return dict(op=op, seqs=seqs, new=new, before=rng.randrange(0, 1000), kv_heads=kv_heads, head=head, block=block, dtype=dtype)
    seqs, length = _log(rng, 1, 64), _log(rng, 64, 32768)
    length = max(64, min(length, MOST_CACHE // (seqs * kv_heads)))
    if op == "attention":
        return dict(op=op, seqs=seqs, length=length, queries=rng.choice([1, 1, 2, 3, 5, 8]), kv_heads=kv_heads,
                    group=rng.choice([1, 2, 4, 5, 8]), head=head, block=block, weights=rng.random() < 0.5, dtype=dtype)
    budget = max(1, int(length * rng.uniform(0.1, 0.9)))
    return dict(op=op, seqs=seqs, length=length, budget=budget, recent=rng.randrange(0, budget + 1),
                kv_heads=kv_heads, head=head, block=block)


# ------------------------------------------------------------------ inputs

def _dtype(case):
    return torch.float16 if case["dtype"] == "f16" else torch.bfloat16


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _lengths(case):
    """Lengths of the sequences: the first is the longest, the others spread below it."""
    L = case["length"]
    return [L - (b * 37) % (L // 2 + 1) for b in range(case["seqs"])]


def _activations(g, tokens, cols, dtype):
    """Normal, with one channel in 200 twenty times as large, as activations have them."""
    x = torch.randn(tokens, cols, generator=g, device=DEV)
    x[:, torch.randperm(cols, generator=g, device=DEV)[:(cols + 199) // 200]] *= 20.0
    return x.to(dtype)


def _weights(g, rows, cols, dtype):
    """N(0, 0.02^2), pruned to two of every four by magnitude."""
    w = torch.randn(rows, cols, generator=g, device=DEV) * 0.02
    n = cols // 4 * 4
    q = w[:, :n].abs().view(rows, n // 4, 4)
    w[:, :n] *= (q >= q.sort(-1).values[..., 2:3]).view(rows, n)
    return w.to(dtype)


def _pool(g, seqs, lengths, kv_heads, head, block, spare=0):
    """An 8-bit cache of random keys and values whose blocks lie in a random order."""
    per = max((n + block - 1) // block for n in lengths) + spare
    n_blocks = seqs * per
    table = torch.randperm(n_blocks, generator=g, device=DEV).view(seqs, per).to(torch.int32)
    codes, scales = [], []
    for _ in range(2):
        x = torch.randn(n_blocks, kv_heads, block, head, generator=g, device=DEV)
        e = _cache_exponent(x.abs().amax((2, 3)))
        s = _pow2(e)
        codes.append((x / s[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8))
        scales.append(s)
    return dict(k=codes[0], v=codes[1], ks=scales[0], vs=scales[1], table=table)


def _empty_pool(seqs, tokens, kv_heads, head, block):
    per = (tokens + block - 1) // block
    shape = (seqs * per, kv_heads, block, head)
    return dict(k=torch.zeros(shape, dtype=torch.uint8, device=DEV), v=torch.zeros(shape, dtype=torch.uint8, device=DEV),
                ks=torch.ones(shape[:2], device=DEV), vs=torch.ones(shape[:2], device=DEV),
                table=torch.arange(seqs * per, device=DEV, dtype=torch.int32).view(seqs, per))


def _handle(pool):
    """The library's handle of a cache, which a program makes once."""
    from paper_2501_16376_b200 import binding as sp
    return sp.KvCache(pool["k"], pool["v"], pool["ks"], pool["vs"], pool["table"])


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    if case["op"] == "quantize":
        s["W"] = _weights(g, case["rows"], case["cols"], _dtype(case))
        s["mask"] = None
        if case["masked"]:                            # a random keep mask of the selection's layout
            words = (case["cols"] + 31) // 32
            m = torch.randint(-2 ** 31, 2 ** 31, (case["rows"], words), generator=g, device=DEV)
            if case["cols"] % 32:
                m[:, -1] &= (1 << (case["cols"] % 32)) - 1
            s["mask"] = m.to(torch.int32)
        s["out"] = torch.empty_like(s["W"])
    elif case["op"] == "linear":
        w = _weights(g, case["rows"], case["cols"], _dtype(case))
        mag, e = _quantize(w.float())
        s["codes"], s["scales"] = _pack(mag, e)
        s["X"] = _activations(g, case["tokens"], case["cols"], _dtype(case))
        s["Y"] = torch.empty(case["tokens"], case["rows"], dtype=_dtype(case), device=DEV)
    elif case["op"] == "append":
        B, n, T = case["seqs"], case["new"], case["block"]
        start = [max(0, case["before"] - 7 * b) for b in range(B)]
        pool = _pool(g, B, [p + n for p in start], case["kv_heads"], case["head"], T)
        s.update(pool, start=torch.tensor(start, dtype=torch.int32, device=DEV))
        shape = (B, n, case["kv_heads"], case["head"])
        s["K"], s["V"] = (torch.randn(shape, generator=g, device=DEV).mul_(1.5).to(_dtype(case)) for _ in range(2))
        if own:
            s["cache"] = _handle(s)
    elif case["op"] == "attention":
        B, H = case["seqs"], case["kv_heads"]
        lens = _lengths(case)
        s.update(_pool(g, B, lens, H, case["head"], case["block"]))
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s["Q"] = torch.randn(B, case["queries"], H * case["group"], case["head"], generator=g, device=DEV).mul_(2.0).to(_dtype(case))
        s["O"] = torch.empty_like(s["Q"])
        s["acc"] = s["acc_out"] = None
        if case["weights"]:
            s["acc"] = torch.rand(B, H, case["length"], generator=g, device=DEV)
            s["acc_out"] = torch.zeros_like(s["acc"])
        if own:
            s["cache"] = _handle(s)
    else:
        B, H = case["seqs"], case["kv_heads"]
        lens = _lengths(case)
        s.update(_pool(g, B, lens, H, case["head"], case["block"]))
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        # accumulated weights fall off steeply: few tokens hold most of them
        s["acc"] = torch.rand(B, H, case["length"], generator=g, device=DEV).pow_(8)
        s["dst"] = _empty_pool(B, case["budget"], H, case["head"], case["block"])
        s["acc_out"] = torch.zeros(B, H, case["budget"], device=DEV)
        s["kept"] = torch.zeros(B, H, case["budget"], dtype=torch.int32, device=DEV)
        s["lens_out"] = torch.zeros(B, dtype=torch.int32, device=DEV)
        if own:
            s["cache"], s["dst_cache"] = _handle(s), _handle(s["dst"])
    return s


# ------------------------------------------------------------------ plain forms

def _pow2(e):
    """2^e in binary32 for whole e from -149 to 127, from its bits."""
    e = e.to(torch.int32)
    small = torch.ones_like(e) << (e + 149).clamp(0, 22)
    return torch.where(e >= -126, (e + 127) << 23, small).view(torch.float32)


def _blocks32(x):
    """[rows, cols] -> [rows, blocks, 32], zeros past the last column."""
    rows, cols = x.shape
    nb = (cols + 31) // 32
    if nb * 32 != cols:
        x = torch.cat([x, x.new_zeros(rows, nb * 32 - cols)], 1)
    return x.view(rows, nb, 32)


def _quantize(x):
    """4-bit codes [rows, blocks, 32] and scale bytes [rows, blocks] of a binary32 matrix."""
    x = _blocks32(x)
    amax = x.abs().amax(-1)
    e = (torch.frexp(amax).exponent - 3).clamp_(min=-127)
    e = torch.where(amax > 0, e, torch.full_like(e, -127))
    # two factors: 2^-e itself may be too large for binary32
    h = torch.div(-e, 2, rounding_mode="floor")
    a = (x.abs() * _pow2(h)[..., None] * _pow2(-e - h)[..., None])
    # steps of 0.5 below 2, 1 below 4, 2 above; ties to the even code
    code = torch.where(a < 2, torch.round(a * 2), torch.where(a < 4, torch.round(a) + 2, torch.round(a / 2) + 4))
    code = code.clamp_(max=7).to(torch.int32) + 8 * torch.signbit(x).to(torch.int32)
    bad = ~torch.isfinite(amax)
    return code.masked_fill_(bad[..., None], 0), (e + 127).masked_fill_(bad, 255).to(torch.int32)


def _values(code, byte):
    """Binary32 values [rows, blocks * 32] of codes and scale bytes."""
    grid = torch.tensor(GRID + tuple(-g for g in GRID), device=code.device)
    v = grid[code.long()] * _pow2(byte.clamp(max=254) - 127)[..., None]
    v = torch.where((byte == 255)[..., None], torch.full_like(v, float("nan")), v)
    return v.reshape(code.shape[0], -1)


def _pack(code, byte):
    """The stored layout of codes and scale bytes."""
    rows, nb = byte.shape
    c = code.view(rows, nb * 16, 2)
    codes = (c[..., 0] | (c[..., 1] << 4)).to(torch.uint8)
    rt, kt = (rows + 127) // 128, (nb + 3) // 4
    t = torch.zeros(rt * 128, kt * 4, dtype=torch.uint8, device=byte.device)
    t[:rows, :nb] = byte.to(torch.uint8)
    scales = t.view(rt, 4, 32, kt, 4).permute(0, 3, 2, 1, 4).reshape(-1)
    return codes, scales.contiguous()


def _unpack(codes, scales, cols):
    rows, nb = codes.shape[0], (cols + 31) // 32
    rt, kt = (rows + 127) // 128, (nb + 3) // 4
    c = codes[:, :nb * 16].to(torch.int32)
    code = torch.stack([c & 15, c >> 4], -1).view(rows, nb, 32)
    byte = scales[:rt * kt * 512].view(rt, kt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rt * 128, kt * 4)
    return code, byte[:rows, :nb].to(torch.int32)


def _mask_bits(mask, cols):
    j = torch.arange(cols, device=mask.device)
    return (mask[:, j // 32] >> (j % 32).to(torch.int32)) & 1


def _plain_quantize(s):
    W = s["W"].float()
    if s["mask"] is not None:
        W = torch.where(_mask_bits(s["mask"], W.shape[1]).bool(), W, torch.zeros_like(W))
    return _values(*_quantize(W))[:, :W.shape[1]].to(s["W"].dtype)


def _plain_linear(s):
    X = s["X"].float()
    if s["case"]["mode"] == "a4":
        X = _values(*_quantize(X))[:, :X.shape[1]]
    W = _values(*_unpack(s["codes"], s["scales"], X.shape[1]))[:, :X.shape[1]]
    return (X @ W.t()).to(s["X"].dtype)


def _cache_exponent(amax):
    """The least e with amax <= 448 * 2^e, at least -126."""
    m, x = torch.frexp(amax)
    e = x - 9 + (m > 0.875).to(x.dtype)
    return torch.where(amax > 0, e, torch.full_like(e, -126)).clamp_(min=-126)


def _encode(x, e):
    """e4m3 of x / 2^e, [..., tokens, head] with e [...]; what is not finite becomes NaN."""
    y = x * _pow2(-e)[..., None, None]
    return torch.where(torch.isfinite(x), y, torch.full_like(y, float("nan"))).to(torch.float8_e4m3fn).view(torch.uint8)


def _append_one(s, codes, scales, new):
    """The touched blocks of one of K, V: [sequences, touched, kv heads, tokens, head]."""
    B, n, H, D = new.shape
    T, start, table = s["case"]["block"], s["start"].long(), s["table"].long()
    touched = (n + T - 2) // T + 1
    first = start // T
    blk = first[:, None] + torch.arange(touched, device=new.device)          # block of the sequence
    pos = blk[..., None] * T + torch.arange(T, device=new.device)            # [B, touched, T]
    t = pos - start[:, None, None]
    is_new, is_old = (t >= 0) & (t < n), t < 0
    b = torch.arange(B, device=new.device)[:, None, None]
    x = new.float()[b, t.clamp(0, n - 1)].permute(0, 1, 3, 2, 4)             # [B, touched, H, T, D]
    fin = torch.where(torch.isfinite(x) & is_new[:, :, None, :, None], x, torch.zeros_like(x))
    live = is_new.any(-1)
    ids = table[b[..., 0], blk.clamp(max=table.shape[1] - 1)]
    old_codes, old_scale = codes[ids], scales[ids]
    e_old = torch.frexp(old_scale).exponent - 1
    e = _cache_exponent(fin.abs().amax((3, 4)))
    e = torch.where(is_old.any(-1)[..., None], torch.maximum(e, e_old), e)
    old = old_codes.view(torch.float8_e4m3fn).float() * old_scale[..., None, None]
    out = torch.where(is_new[:, :, None, :, None], _encode(x, e),
                      torch.where(is_old[:, :, None, :, None], _encode(old, e), old_codes))
    codes[ids[live]] = out[live]
    scales[ids[live]] = _pow2(e)[live]


def _plain_append(s):
    _append_one(s, s["k"], s["ks"], s["K"])
    _append_one(s, s["v"], s["vs"], s["V"])
    return s["k"].view(torch.float8_e4m3fn), s["v"].view(torch.float8_e4m3fn), s["ks"], s["vs"]


def _dense(codes, scales, table, length, as_type=torch.float32):
    """[sequences, kv heads, length, head] values of a cache's first tokens."""
    v = codes[table.long()].view(torch.float8_e4m3fn).to(as_type) * scales[table.long()].to(as_type)[..., None, None]
    B, nb, H, T, D = v.shape
    return v.permute(0, 2, 1, 3, 4).reshape(B, H, nb * T, D)[:, :, :length]


def _plain_attention(s):
    c = s["case"]
    L, n, G, H = c["length"], c["queries"], c["group"], c["kv_heads"]
    B, D = c["seqs"], c["head"]
    K, V = _dense(s["k"], s["ks"], s["table"], L), _dense(s["v"], s["vs"], s["table"], L)
    Q = s["Q"].float().view(B, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, n * G, D)
    S = (Q @ K.transpose(2, 3)) / math.sqrt(D)
    at = s["lens"].long()[:, None] - n + torch.arange(n, device=Q.device)     # position of a query
    j = torch.arange(L, device=Q.device)
    seen = (j <= at[..., None])[:, None].repeat_interleave(G, 2)              # [B, 1, n G, L]
    S = torch.where(seen, S, torch.full_like(S, float("-inf")))
    top = S.amax(-1, keepdim=True)
    P = torch.where(seen, torch.exp(S - top), torch.zeros_like(S))
    total = P.sum(-1, keepdim=True)
    P = torch.where(total > 0, P / total, torch.zeros_like(P))
    in_len = (j < s["lens"].long()[:, None])[:, None, :, None]
    O = P @ torch.where(in_len, V, torch.zeros_like(V))
    O = O.view(B, H, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, H * G, D).to(s["Q"].dtype)
    if s["acc"] is None:
        return O
    old = torch.where((j < s["lens"].long()[:, None] - n)[:, None], s["acc"], torch.zeros_like(s["acc"]))
    acc = torch.where((j < s["lens"].long()[:, None])[:, None], old + P.sum(2), torch.zeros_like(old))
    return O, acc


def _select(s):
    """Kept token indices [sequences, kv heads, budget] in their order, -1 past the last."""
    c = s["case"]
    L, budget, recent = c["length"], c["budget"], c["recent"]
    n = s["lens"].long()[:, None, None]
    j = torch.arange(L, device=DEV)
    m = n.clamp(max=budget)
    key = s["acc"] + 0.0
    key = torch.where(torch.isnan(key) | (j >= n - m.clamp(max=recent)), torch.full_like(key, float("inf")), key)
    key = torch.where(j < n, key, torch.full_like(key, float("-inf")))
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :budget]
    slot = torch.arange(budget, device=DEV)
    order = torch.where(slot < m, order, torch.full_like(order, L)).sort(-1).values
    return torch.where(order < L, order, torch.full_like(order, -1))


def _plain_evict(s):
    c, T = s["case"], s["case"]["block"]
    kept = _select(s)
    B, H, m = kept.shape
    nb = (m + T - 1) // T
    pad = torch.full((B, H, nb * T), -1, device=DEV, dtype=kept.dtype)
    pad[..., :m] = kept
    at = pad.clamp(min=0)
    ids = s["table"].long()[torch.arange(B, device=DEV)[:, None, None], at // T]
    h = torch.arange(H, device=DEV)[None, :, None]
    live = (pad >= 0).view(B, H, nb, T)
    to = s["dst"]["table"].long()[:, :nb]                                     # [B, nb]
    for codes, scales, out, out_scale in ((s["k"], s["ks"], s["dst"]["k"], s["dst"]["ks"]),
                                          (s["v"], s["vs"], s["dst"]["v"], s["dst"]["vs"])):
        x = codes[ids, h, at % T].view(torch.float8_e4m3fn).float() * scales[ids, h][..., None]
        x = x.view(B, H, nb, T, -1)
        x = torch.where(live[..., None], x, torch.zeros_like(x))
        fin = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
        e = _cache_exponent(fin.abs().amax((3, 4)))                           # [B, H, nb]
        out[to] = _encode(x, e).transpose(1, 2)
        out_scale[to] = _pow2(e).transpose(1, 2)
    acc = torch.where(kept >= 0, s["acc"].gather(2, kept.clamp(min=0)), torch.zeros_like(s["acc_out"]))
    d = s["dst"]
    return (kept.to(torch.int32), acc, s["lens"].clamp(max=c["budget"]), d["k"].view(torch.float8_e4m3fn),
            d["v"].view(torch.float8_e4m3fn), d["ks"], d["vs"])


PLAIN = dict(quantize=_plain_quantize, linear=_plain_linear, append=_plain_append,
             attention=_plain_attention, evict=_plain_evict)


# ------------------------------------------------------------------ the library's calls

def _own_quantize(sp, s):
    codes, scales = sp.sp_mx4_quantize(s["W"], mask=s["mask"])
    return sp.sp_mx4_dequantize(codes, scales, s["W"].shape[1], W_out=s["out"])


def _own_linear(sp, s):
    mode = sp.SP_MX4_A4 if s["case"]["mode"] == "a4" else sp.SP_MX4_A16
    return sp.sp_mx4_linear(s["X"], s["codes"], s["scales"], mode=mode, Y=s["Y"])


def _own_append(sp, s):
    s["cache"].sp_cache_append(s["K"], s["V"], s["start"])
    return s["k"].view(torch.float8_e4m3fn), s["v"].view(torch.float8_e4m3fn), s["ks"], s["vs"]


def _own_attention(sp, s):
    O = s["cache"].sp_cache_attention(s["Q"], s["lens"], s["case"]["length"], O=s["O"],
                                      acc_in=s["acc"], acc_out=s["acc_out"])
    return O if s["acc"] is None else (O, s["acc_out"])


def _own_evict(sp, s):
    c, d = s["case"], s["dst"]
    s["cache"].sp_cache_evict(s["lens"], c["length"], s["acc"], c["budget"], c["recent"], s["dst_cache"],
                              acc_out=s["acc_out"], kept_out=s["kept"], lens_out=s["lens_out"])
    return (s["kept"], s["acc_out"], s["lens_out"], d["k"].view(torch.float8_e4m3fn),
            d["v"].view(torch.float8_e4m3fn), d["ks"], d["vs"])


OWN = dict(quantize=_own_quantize, linear=_own_linear, append=_own_append,
           attention=_own_attention, evict=_own_evict)


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2501_16376_b200 import binding as sp
        return OWN[op](sp, state)
    return PLAIN[op](state)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        blocks = case["rows"] * ((case["cols"] + 31) // 32)
        return dict(bytes=n * 4 + blocks * 17 + (n // 8 if case["masked"] else 0), flops=0)
    if case["op"] == "linear":
        t, c, r = case["tokens"], case["cols"], case["rows"]
        return dict(bytes=r * ((c + 31) // 32) * 17 + 2 * t * (c + r), flops=2 * t * c * r)
    H, D = case["kv_heads"], case["head"]
    if case["op"] == "append":
        n = case["seqs"] * case["new"] * H * D
        return dict(bytes=2 * n * 3, flops=0)
    total = sum(_lengths(case))
    if case["op"] == "attention":
        heads, n = H * case["group"], case["queries"]
        io = 2 * 2 * case["seqs"] * n * heads * D
        w = 8 * total * H if case["weights"] else 0
        return dict(bytes=total * H * D * 2 + io + w, flops=4 * n * heads * D * total)
    kept = sum(min(n, case["budget"]) for n in _lengths(case))
    return dict(bytes=total * H * 4 + kept * H * (2 * 2 * D + 8), flops=0)


# ------------------------------------------------------------------ 64-bit values

def _two(e):
    """2^e in binary64 for whole e, from its bits."""
    return ((torch.round(e.double()).long() + 1023) << 52).view(torch.float64)


def _exact_mx4(x):
    """Nearest 4-bit values, in binary64, by distance to every value of the grid."""
    rows, cols = x.shape
    nb = (cols + 31) // 32
    p = torch.zeros(rows, nb * 32, dtype=torch.float64, device=x.device)
    p[:, :cols] = x.double()
    p = p.view(rows, nb, 32)
    amax = p.abs().amax(-1, keepdim=True)
    e = torch.where(amax > 0, torch.floor(torch.log2(amax.clamp(min=2.0 ** -1000))) - 2, amax)
    e = torch.where(amax >= _two(e + 3), e + 1, torch.where(amax < _two(e + 2), e - 1, e)).clamp(min=-127)
    a = p.abs() / _two(e)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    best = torch.zeros_like(a)
    dist = torch.full_like(a, float("inf"))
    for i in (0, 2, 4, 6, 1, 3, 5, 7):                # even codes first: a tie stays with them
        d = (a - grid[i]).abs()
        closer = d < dist
        best, dist = torch.where(closer, grid[i], best), torch.where(closer, d, dist)
    return (best * torch.sign(p) * _two(e)).view(rows, nb * 32)[:, :cols]


def _exact_cache(s, which, b, n):
    """[kv heads, n, head] binary64 values of the first n tokens of sequence b."""
    T = s["case"]["block"]
    ids = s["table"][b, :(n + T - 1) // T].long()
    x = s[which][ids].view(torch.float8_e4m3fn).double() * s[which + "s"][ids].double()[:, :, None, None]
    return x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :n]


def _exact_exponent(amax):
    """The least e with amax <= 448 * 2^e, at least -126, in binary64."""
    e = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -200) / 448)).clamp(min=-126)
    return torch.where(amax > 448 * _two(e), e + 1, torch.where((amax <= 448 * _two(e - 1)) & (e > -126), e - 1, e))


def _exact_e4m3(x):
    """The nearest value with 3 bits after the leading one, steps of 2^-9 at the least."""
    step = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = _two(torch.where(x.abs() >= _two(step + 1), step + 1, step) - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        W = s["W"].double()
        if s["mask"] is not None:
            for j in range(W.shape[1]):
                W[:, j] *= (s["mask"][:, j // 32] >> (j % 32)) & 1
        return _exact_mx4(W)
    if case["op"] == "linear":
        X = s["X"].double() if case["mode"] == "a16" else _exact_mx4(s["X"])
        rows, cols = case["rows"], case["cols"]
        nb, kt = (cols + 31) // 32, ((cols + 31) // 32 + 3) // 4
        r = torch.arange(rows, device=DEV)[:, None]
        q = torch.arange(nb, device=DEV)[None]
        byte = s["scales"][(r // 128 * kt + q // 4) * 512 + r % 32 * 16 + r // 32 % 4 * 4 + q % 4].double()
        W = torch.empty(rows, nb * 32, dtype=torch.float64, device=DEV)
        grid = torch.tensor(GRID + tuple(-v for v in GRID), dtype=torch.float64, device=DEV)
        W[:, 0::2] = grid[(s["codes"][:, :nb * 16] & 15).long()]
        W[:, 1::2] = grid[(s["codes"][:, :nb * 16] >> 4).long()]
        W = (W.view(rows, nb, 32) * _two(byte - 127)[..., None]).view(rows, -1)[:, :cols]
        return X @ W.t()
    B, H, D = case["seqs"], case["kv_heads"], case["head"]
    if case["op"] == "append":
        pools = {w: s[w].view(torch.float8_e4m3fn).double() for w in ("k", "v")}
        scale = {w: s[w + "s"].double() for w in ("k", "v")}
        T = case["block"]
        for b, start in enumerate(s["start"].tolist()):
            for i in range(start // T, (start + case["new"] - 1) // T + 1):
                block, lo, hi = int(s["table"][b, i]), max(start, i * T), min(start + case["new"], (i + 1) * T)
                for w in ("k", "v"):
                    x = s[w.upper()][b, lo - start:hi - start].double().transpose(0, 1)      # [H, tokens, D]
                    e = _exact_exponent(x.abs().amax((1, 2)))
                    if lo > i * T:
                        was = torch.round(torch.log2(scale[w][block]))
                        e = torch.maximum(e, was)
                        old = pools[w][block, :, :lo - i * T]
                        pools[w][block, :, :lo - i * T] = _exact_e4m3(old * _two(was - e)[:, None, None])
                    pools[w][block, :, lo - i * T:hi - i * T] = _exact_e4m3(x / _two(e)[:, None, None])
                    scale[w][block] = _two(e)
        return pools["k"], pools["v"], scale["k"], scale["v"]
    if case["op"] == "evict":
        budget, T = case["budget"], case["block"]
        nb = (budget + T - 1) // T
        d = s["dst"]
        pools = {w: d[w].view(torch.float8_e4m3fn).double() for w in ("k", "v")}
        scale = {w: d[w + "s"].double() for w in ("k", "v")}
        kept = torch.full((B, H, budget), -1, dtype=torch.int64, device=DEV)
        acc = torch.zeros(B, H, budget, dtype=torch.float64, device=DEV)
        for b, length in enumerate(_lengths(case)):
            m = min(length, budget)
            free = length - min(case["recent"], m)                           # tokens the weights decide on
            for h in range(H):
                a = s["acc"][b, h, :free].double()
                cut = torch.sort(a, descending=True).values[m - (length - free) - 1] if m > length - free else math.inf
                over, ties = (a > cut).nonzero()[:, 0], (a == cut).nonzero()[:, 0]
                chosen = torch.cat([over, ties[:m - (length - free) - over.numel()],
                                    torch.arange(free, length, device=DEV)]).sort().values
                kept[b, h, :m] = chosen
                acc[b, h, :m] = s["acc"][b, h, chosen].double()
            for w in ("k", "v"):
                dense = torch.zeros(H, nb * T, D, dtype=torch.float64, device=DEV)
                dense[:, :m] = _exact_cache(s, w, b, length).gather(1, kept[b, :, :m, None].expand(H, m, D))
                dense = dense.view(H, nb, T, D).transpose(0, 1)
                e = _exact_exponent(dense.abs().amax((2, 3)))
                to = d["table"][b, :nb].long()
                pools[w][to] = _exact_e4m3(dense / _two(e)[..., None, None])
                scale[w][to] = _two(e)
        return kept, acc, None, pools["k"], pools["v"], scale["k"], scale["v"]
    n, G = case["queries"], case["group"]
    out = torch.zeros(B, n, H * G, D, dtype=torch.float64, device=DEV)
    acc = torch.zeros(B, H, case["length"], dtype=torch.float64, device=DEV)
    for b, length in enumerate(_lengths(case)):
        K, V = _exact_cache(s, "k", b, length), _exact_cache(s, "v", b, length)
        if case["weights"]:
            acc[b, :, :max(0, length - n)] = s["acc"][b, :, :max(0, length - n)].double()
        for i in range(n):
            end = length - n + i + 1
            if end < 1:
                continue
            q = s["Q"][b, i].double().view(H, G, D)
            p = torch.softmax(q @ K[:, :end].transpose(1, 2) / math.sqrt(D), -1)
            out[b, i] = (p @ V[:, :end]).view(H * G, D)
            acc[b, :, :end] += p.sum(1)
    return (out, acc) if case["weights"] else out
