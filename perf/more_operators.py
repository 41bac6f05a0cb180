"""Measured cases of the operators that serve several answers of one prompt: positions (norms of
queries and keys with the rotation), the pages of the 8-bit cache (fork, reserve, compact), and
attention over a prefix that a group of sequences shares.

Head counts and sizes are those of the models the package prunes (LLaMA-3-8B: 32 heads over 8 kv
heads of 128; LLaMA-2-7B: 32 of 128; LLaMA-2-13B: 40 of 128; Pythia-410M: 16 of 64).

``run`` computes an operator from elementary torch operations in binary32 (angles in binary64), or,
with ``own`` set, calls the library.  The cache is the library's: e4m3 codes [blocks, kv heads,
tokens of a block, head size] and binary32 power-of-two scales [blocks, kv heads], for K and for V;
a table [sequences, blocks] names the blocks, -1 none; refs [blocks] counts the table entries that
name a block.
"""
import math

import torch

own = False

DEV = "cuda"
MOST_ROTARY = 32768 * 40 * 128                       # values of the largest listed rotation
MOST_SHARED = 8 * 32 * 4 * 8 * 8191 * 128            # (row, kv head, token, channel) of the largest prefix
MOST_TAIL = 8 * 32 * 8 * 512                         # (sequence, kv head, token) of the largest tails
MOST_CACHE = 8 * 8 * 8191 * 4                        # (group, kv head, token) of the largest prefixes
MOST_POOL = 8192 * 8 * 32 * 128                       # values of K in the largest listed pool


def listed():
    return [
        # a decoding step of 8 sequences of LLaMA-3-8B's heads, normalised: all launch and latency
        dict(name="rotary 8x1 bf16 normed", op="rotary", seqs=8, tokens=1, heads=32, kv_heads=8, head=128, rotary=128, pairs=False, norm=True, fused=True, far=8000, theta=500000.0, dtype="bf16"),
        # ragged prompts of Pythia-410M, which rotates a quarter of its head and normalises nothing
        dict(name="rotary 4x2047 f16 quarter", op="rotary", seqs=4, tokens=2047, heads=16, kv_heads=16, head=64, rotary=16, pairs=False, norm=False, fused=True, far=0, theta=10000.0, dtype="f16"),
        # a long document at far positions, neighbouring values turned together
        dict(name="rotary 1x32768 bf16 normed pairs", op="rotary", seqs=1, tokens=32768, heads=32, kv_heads=8, head=128, rotary=128, pairs=True, norm=True, fused=False, far=1000000, theta=500000.0, dtype="bf16"),
        # four answers of a short prompt, Pythia-410M, their first blocks
        dict(name="fork 1 to 4", op="fork", groups=1, size=4, length=517, kv_heads=16, head=64, block=16, new=1),
        # 64 answers of four prompts of LLaMA-3-8B
        dict(name="fork 4 to 64", op="fork", groups=4, size=16, length=4095, kv_heads=8, head=128, block=32, new=1),
        # many answers with the widest cache (LLaMA-2-7B), a chunk of tokens ahead
        dict(name="fork 8 to 128 wide", op="fork", groups=8, size=16, length=1001, kv_heads=32, head=128, block=64, new=32),
        # a small pool after a few answers have ended
        dict(name="compact 300 blocks", op="compact", blocks=300, seqs=8, live=0.4, kv_heads=16, head=64, block=16),
        # a pool of half a gigabyte, a third of it in use
        dict(name="compact 8192 blocks", op="compact", blocks=8192, seqs=64, live=0.35, kv_heads=8, head=128, block=32),
        # four short answers, one token
        dict(name="shared 4 of 517 f16", op="shared", groups=1, size=4, prefix=517, tail=5, queries=1, kv_heads=16, group=1, head=64, block=16, dtype="f16"),
        # 16 answers of a prompt of LLaMA-3-8B, two tokens at once
        dict(name="shared 16 of 4095 q2 bf16", op="shared", groups=1, size=16, prefix=4095, tail=200, queries=2, kv_heads=8, group=4, head=128, block=32, dtype="bf16"),
        # 64 answers of a long prompt of LLaMA-2-13B (40 heads, no groups)
        dict(name="shared 64 of 8191 f16", op="shared", groups=1, size=64, prefix=8191, tail=77, queries=1, kv_heads=40, group=1, head=128, block=64, dtype="f16"),
        # the largest batch: 8 prompts with 32 answers each
        dict(name="shared 8x32 of 8191 bf16", op="shared", groups=8, size=32, prefix=8191, tail=300, queries=1, kv_heads=8, group=4, head=128, block=32, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotary", "rotary", "fork", "compact", "shared", "shared", "shared"])
    dtype = rng.choice(["f16", "bf16"])
    kv_heads, head, block = rng.choice([1, 2, 5, 8, 16, 32, 40]), rng.choice([64, 128]), rng.choice([16, 32, 64])
    if op == "rotary":
        kv_heads, group = rng.choice([1, 2, 5, 8, 16]), rng.choice([1, 2, 4, 5])
        seqs, tokens = _log(rng, 1, 64), _log(rng, 1, 32768)
        tokens = max(1, min(tokens, MOST_ROTARY // (seqs * kv_heads * (group + 1) * head)))
        return dict(op=op, seqs=seqs, tokens=tokens, heads=kv_heads * group, kv_heads=kv_heads, head=head,
                    rotary=rng.choice([head, head, head // 2, head // 4, 24]), pairs=rng.random() < 0.4,
                    norm=rng.random() < 0.6, fused=rng.random() < 0.5, far=rng.choice([0, 1000, 100000, 1000000]),
                    theta=rng.choice([10000.0, 500000.0]), dtype=dtype)
    if op == "fork":
        groups, size, length = _log(rng, 1, 8), _log(rng, 1, 16), _log(rng, 16, 4096)
        length = max(16, min(length, MOST_POOL // (groups * kv_heads * head) - size * 100))
        return dict(op=op, groups=groups, size=size, length=length, kv_heads=kv_heads, head=head, block=block, new=rng.choice([1, 1, 3, 32]))
    if op == "compact":
        blocks = max(8, min(_log(rng, 8, 8192), MOST_POOL // (kv_heads * head * block)))
        return dict(op=op, blocks=blocks, seqs=_log(rng, 1, 64), live=round(rng.uniform(0.05, 0.95), 2), kv_heads=kv_heads, head=head, block=block)
    groups, size, queries, group = _log(rng, 1, 8), _log(rng, 1, 64), rng.choice([1, 1, 1, 2, 4]), rng.choice([1, 2, 4, 5, 8])
    tail = max(queries, min(_log(rng, 1, 1024), MOST_TAIL // (groups * size * kv_heads)))
    prefix = _log(rng, 16, 16384)
    prefix = max(16, min(prefix, MOST_SHARED // (groups * size * queries * group * kv_heads * head), MOST_CACHE // (groups * kv_heads)))
    return dict(op=op, groups=groups, size=size, prefix=prefix, tail=tail, queries=queries, kv_heads=kv_heads,
                group=group, head=head, block=block, dtype=dtype)


# ------------------------------------------------------------------ inputs

def _dtype(case):
    return torch.float16 if case["dtype"] == "f16" else torch.bfloat16


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _prefixes(case):
    """Prefix lengths of the groups: the first is the longest, the others a little shorter."""
    P = case["prefix"]
    return [P - (g * 37) % (P // 4 + 1) for g in range(case["groups"])]


def _shared_tokens(case):
    """Of each prefix, what lies in whole blocks: those the sequences of a group share."""
    return [p // case["block"] * case["block"] for p in _prefixes(case)]


def _lengths(case):
    """Lengths of all sequences: the prefix and 1 to ``tail`` tokens of the sequence's own."""
    own_tokens = lambda b: max(case["queries"], case["tail"] - (b * 13) % (case["tail"] // 2 + 1))
    return [p + own_tokens(g * case["size"] + i) for g, p in enumerate(_prefixes(case)) for i in range(case["size"])]


def _codes(g, blocks, kv_heads, block, head):
    """e4m3 codes and scales of random keys or values."""
    x = torch.randn(blocks, kv_heads, block, head, generator=g, device=DEV)
    m, e = torch.frexp(x.abs().amax((2, 3)))
    s = torch.exp2((e - 9 + (m > 0.875).to(e.dtype)).float())
    return (x / s[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8), s


def _pool(s, g, blocks, case):
    s["k"], s["ks"] = _codes(g, blocks, case["kv_heads"], case["block"], case["head"])
    s["v"], s["vs"] = _codes(g, blocks, case["kv_heads"], case["block"], case["head"])


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _handle(s):
    """The library's handle of a cache, which a program makes once."""
    from paper_2501_16376_b200 import binding as sp
    return sp.KvCache(s["k"], s["v"], s["ks"], s["vs"], s["table"], refs=s.get("refs"))


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    if case["op"] == "rotary":
        B, n, H, Hk, D = case["seqs"], case["tokens"], case["heads"], case["kv_heads"], case["head"]
        if case["fused"]:                              # views of one projection's output
            x = torch.randn(B, n, H + 2 * Hk, D, generator=g, device=DEV).mul_(1.5).to(_dtype(case))
            s["Q"], s["K"] = x[:, :, :H], x[:, :, H:H + Hk]
        else:
            s["Q"], s["K"] = (torch.randn(B, n, h, D, generator=g, device=DEV).mul_(1.5).to(_dtype(case)) for h in (H, Hk))
        s["wq"] = s["wk"] = None
        if case["norm"]:
            s["wq"], s["wk"] = ((1 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(_dtype(case)) for _ in range(2))
        s["start"] = (case["far"] + torch.randint(0, 1000, (B,), generator=g, device=DEV)).to(torch.int32)
        s["freq"] = (case["theta"] ** (-torch.arange(0, case["rotary"], 2, device=DEV, dtype=torch.float64) / case["rotary"])).float()
        s["Qo"], s["Ko"] = (torch.empty(B, n, h, D, dtype=_dtype(case), device=DEV) for h in (H, Hk))
    elif case["op"] == "fork":
        # every group's first row holds a prompt in blocks of its own; the other rows are empty
        n, T = case["size"], case["block"]
        B, per = case["groups"] * n, (case["length"] + T - 1) // T
        cols = (case["length"] + case["new"] + T - 1) // T
        more = B * (cols - case["length"] // T)        # blocks that the new tokens may ask for
        blocks = case["groups"] * per + more + 5
        _pool(s, g, blocks, case)
        ids = torch.randperm(blocks, generator=g, device=DEV)[:case["groups"] * per].view(case["groups"], per).to(torch.int32)
        s["table"] = torch.full((B, cols), -1, dtype=torch.int32, device=DEV)
        s["table"][::n, :per] = ids
        s["refs"] = torch.zeros(blocks, dtype=torch.int32, device=DEV)
        s["refs"][ids.long().flatten()] = 1
        rows = [b for b in range(B) if b % n]
        s["dst"], s["src"] = _int32(rows), _int32([b // n * n for b in rows])
        s["start"] = _int32([case["length"]] * B)
        s["status"] = torch.zeros(2, dtype=torch.int32, device=DEV)
        if own:
            s["cache"] = _handle(s)
    elif case["op"] == "compact":
        blocks, B = case["blocks"], case["seqs"]
        _pool(s, g, blocks, case)
        live = max(1, int(blocks * case["live"]))
        ids = torch.randperm(blocks, generator=g, device=DEV)[:live].to(torch.int32)
        per = (live + B - 1) // B
        s["table"] = torch.full((B, per + 3), -1, dtype=torch.int32, device=DEV)
        flat = torch.full((B * per,), -1, dtype=torch.int32, device=DEV)
        flat[:live] = ids
        s["table"][:, :per] = flat.view(B, per)
        if B > 1:                                      # the second row shares the first one's blocks too
            s["table"][1, :per] = s["table"][0, :per]
        named = s["table"].flatten().long()
        s["refs"] = torch.zeros(blocks, dtype=torch.int32, device=DEV)
        s["refs"].scatter_add_(0, named.clamp(min=0), (named >= 0).to(torch.int32))
        s["table_out"], s["refs_out"] = torch.empty_like(s["table"]), torch.empty_like(s["refs"])
        s["live"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        if own:
            s["cache"] = _handle(s)
    else:
        n, T, H = case["size"], case["block"], case["kv_heads"]
        B, shared, lens = case["groups"] * case["size"], _shared_tokens(case), _lengths(case)
        first = [sum(shared[:i]) // T for i in range(len(shared))]
        cols = max((x + T - 1) // T for x in lens)
        table, at = torch.full((B, cols), -1, dtype=torch.int32), sum(shared) // T
        for b, length in enumerate(lens):
            k, m = shared[b // n] // T, (length + T - 1) // T
            table[b, :k] = torch.arange(first[b // n], first[b // n] + k)
            table[b, k:m] = torch.arange(at, at + m - k)
            at += m - k
        _pool(s, g, at, case)
        order = torch.randperm(at, generator=g, device=DEV).to(torch.int32)
        table = table.to(DEV)
        s["table"] = torch.where(table >= 0, order[table.long().clamp(min=0)], table)
        s["lens"], s["prefix"] = _int32(lens), _int32(_prefixes(case))
        s["group_start"] = _int32([i * n for i in range(case["groups"] + 1)])
        s["Q"] = torch.randn(B, case["queries"], H * case["group"], case["head"], generator=g, device=DEV).mul_(2.0).to(_dtype(case))
        s["O"] = torch.empty_like(s["Q"])
        if own:
            s["cache"] = _handle(s)
    return s


# ------------------------------------------------------------------ plain forms

def _turn(x, w, c, angle, eps=1e-6):
    """x [B, n, heads, D] normalised by head and turned by angle [B, n, rotary / 2]."""
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + eps) * w.float()
    r = c["rotary"]
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    if c["pairs"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _plain_rotary(s):
    place = s["start"].long()[:, None] + torch.arange(s["case"]["tokens"], device=DEV)
    angle = place[..., None].double() * s["freq"].double()
    return _turn(s["Q"], s["wq"], s["case"], angle), _turn(s["K"], s["wk"], s["case"], angle)


def _plain_fork(s):
    c, table, refs = s["case"], s["table"], s["refs"]
    T, new, blocks, one = c["block"], c["new"], refs.numel(), torch.ones_like
    # the rows dst become those of src; the counts follow
    if s["dst"].numel():
        dst, src = s["dst"].long(), s["src"].long()
        was, now = table[dst].flatten().long(), table[src].flatten().long()
        refs.scatter_add_(0, was.clamp(min=0), -(was >= 0).to(torch.int32))
        refs.scatter_add_(0, now.clamp(min=0), (now >= 0).to(torch.int32))
        table[dst] = table[src]
    # requests: the blocks of the new places, in the order of sequences and places
    start = s["start"].long()[:, None]
    place = start // T + torch.arange((new + T - 2) // T + 1, device=DEV)                 # [B, most blocks]
    asked = (place * T < start + new) & (place < table.shape[1])
    at = place.clamp(max=table.shape[1] - 1)
    was = table.gather(1, at).long()
    named = asked & (was >= 0)
    w = was.clamp(min=0)
    count = torch.zeros_like(refs).scatter_add_(0, w.flatten(), named.flatten().to(torch.int32))
    index = torch.arange(asked.numel(), device=DEV).view(asked.shape)
    first = torch.full((blocks,), asked.numel(), device=DEV)
    first.scatter_reduce_(0, w.flatten(), torch.where(named, index, asked.numel()).flatten(), "amin")
    # a block that all its sharers ask for stays with the first of them
    keep = named & ((refs[w] <= 1) | ((count[w] >= refs[w]) & (first[w] == index)))
    need = asked & ~keep
    rank = need.flatten().cumsum(0).view(need.shape) - 1
    free = torch.sort((refs > 0).to(torch.int8), stable=True).indices                     # free ones first, ascending
    n_need, n_free = need.sum(), (refs == 0).sum()
    need = need & (n_need <= n_free)
    to = free[rank.clamp(0, blocks - 1)]
    table.scatter_(1, at, torch.where(need, to, torch.where(asked, was, table.gather(1, at).long())).to(torch.int32))
    copied = need & named & (place == start // T) & (start % T > 0)
    source, target = torch.where(copied, was, to)[copied], to[copied]
    for t in (s["k"], s["v"], s["ks"], s["vs"]):
        t[target] = t[source]
    refs.scatter_add_(0, w.flatten(), -(need & named).flatten().to(torch.int32))
    refs.scatter_add_(0, to.flatten(), need.flatten().to(torch.int32))
    s["status"][0] = torch.clamp(n_need - n_free, min=0)
    s["status"][1] = n_free - torch.where(n_need <= n_free, n_need, torch.zeros_like(n_need))
    return table, refs, s["status"], s["k"], s["v"], s["ks"], s["vs"]


def _plain_compact(s):
    table, refs = s["table"], s["refs"]
    live = refs > 0
    n = live.sum()
    index = torch.arange(refs.numel(), device=DEV)
    holes = (~live & (index < n)).nonzero()[:, 0]
    movers = (live & (index >= n)).nonzero()[:, 0]
    for t in (s["k"], s["v"], s["ks"], s["vs"]):
        t[holes] = t[movers]
    remap = torch.where(live, index, torch.full_like(index, -1))
    remap[movers] = holes
    named = table >= 0
    s["table_out"].copy_(torch.where(named, remap[table.long().clamp(min=0)].to(torch.int32), table))
    out = torch.where(index < n, refs, torch.zeros_like(refs))
    out[holes] = refs[movers]
    s["refs_out"].copy_(out)
    s["live"].copy_(n)
    return s["table_out"], s["refs_out"], s["live"], s["k"], s["v"], s["ks"], s["vs"]


def _dense(s, which, ids):
    """[rows, kv heads, tokens, head] values of the blocks ids [rows, blocks]."""
    v = s[which][ids].view(torch.float8_e4m3fn).float() * s[which + "s"][ids][..., None, None]
    R, nb, H, T, D = v.shape
    return v.permute(0, 2, 1, 3, 4).reshape(R, H, nb * T, D)


def _plain_shared(s):
    c = s["case"]
    n, T, H, G, q, D = c["size"], c["block"], c["kv_heads"], c["group"], c["queries"], c["head"]
    N, B, table, lens = c["groups"], c["groups"] * c["size"], s["table"].long(), s["lens"].long()
    shared = s["prefix"].long() // T                                                      # blocks
    pb = c["prefix"] // T
    tb = (c["tail"] + T - 2 + T) // T                                                     # blocks of the longest tail
    place = lens[:, None] - q + torch.arange(q, device=DEV)                               # [B, q]
    Q = s["Q"].float().view(B, q, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, q * G, D) / math.sqrt(D)
    # the prefix: the queries of a group as rows over its first sequence's blocks
    own_block = shared.repeat_interleave(n)[:, None] + torch.arange(tb, device=DEV)       # [B, tb]
    ids = table.gather(1, own_block.clamp(max=table.shape[1] - 1)).clamp(min=0)
    K, V = _dense(s, "k", ids), _dense(s, "v", ids)
    at = own_block[:, :1, None] * T + torch.arange(tb * T, device=DEV)                    # [B, 1, tb T]
    seen = (at <= place[..., None]).repeat_interleave(G, 1)[:, None]                      # [B, 1, q G, tb T]
    S = torch.where(seen, Q @ K.transpose(2, 3), float("-inf"))
    inside = (at < lens[:, None, None])[..., None]
    V = torch.where(inside, V, 0.0)
    if pb > 0:
        ids = table[::n, :pb].clamp(min=0)
        Kp, Vp = _dense(s, "k", ids), _dense(s, "v", ids)
        rows = Q.view(N, n, H, q * G, D).transpose(1, 2).reshape(N, H, n * q * G, D)
        Sp = rows @ Kp.transpose(2, 3)
        token = torch.arange(pb * T, device=DEV)
        live = token < shared[:, None] * T                                                # [N, pb T]
        sees = live[:, None] & (token <= place.view(N, n * q, 1))
        sees = sees.view(N, n, q, -1).repeat_interleave(G, 2).view(N, 1, n * q * G, -1)
        Sp = torch.where(sees, Sp, float("-inf"))
        Vp = torch.where(live[:, None, :, None], Vp, 0.0)
        top = Sp.amax(-1).view(N, H, n, q * G).transpose(1, 2).reshape(B, H, q * G, 1)
        top = torch.maximum(top, S.amax(-1, keepdim=True))
        P = torch.where(seen, torch.exp(S - top), 0.0)
        rows_top = top.view(N, n, H, q * G).transpose(1, 2).reshape(N, H, n * q * G, 1)
        Pp = torch.where(sees, torch.exp(Sp - rows_top), 0.0)
        back = lambda t: t.view(N, H, n, q * G, -1).transpose(1, 2).reshape(B, H, q * G, -1)
        total = P.sum(-1, keepdim=True) + back(Pp.sum(-1, keepdim=True))
        O = P @ V + back(Pp @ Vp)
    else:
        P = torch.where(seen, torch.exp(S - S.amax(-1, keepdim=True)), 0.0)
        total, O = P.sum(-1, keepdim=True), P @ V
    O = torch.where(total > 0, O / total, 0.0)
    return O.view(B, H, q, G, D).permute(0, 2, 1, 3, 4).reshape(B, q, H * G, D).to(s["Q"].dtype)


PLAIN = dict(rotary=_plain_rotary, fork=_plain_fork, compact=_plain_compact, shared=_plain_shared)


# ------------------------------------------------------------------ the library's calls

def _own_rotary(sp, s):
    return sp.sp_qk_norm_rotary(s["Q"], s["K"], s["start"], s["freq"], q_weight=s["wq"], k_weight=s["wk"],
                                eps=1e-6, pairs=s["case"]["pairs"], Q_out=s["Qo"], K_out=s["Ko"])


def _own_fork(sp, s):
    cache = s["cache"]
    cache.sp_cache_fork(s["dst"], s["src"])
    cache.sp_cache_reserve(s["start"], s["case"]["new"], status=s["status"])
    return s["table"], s["refs"], s["status"], s["k"], s["v"], s["ks"], s["vs"]


def _own_compact(sp, s):
    s["cache"].sp_cache_compact(s["live"], table_out=s["table_out"], refs_out=s["refs_out"])
    return s["table_out"], s["refs_out"], s["live"], s["k"], s["v"], s["ks"], s["vs"]


def _own_shared(sp, s):
    c = s["case"]
    return s["cache"].sp_cache_attention_shared(s["Q"], s["lens"], c["prefix"] + max(c["tail"], c["queries"]),
                                                s["group_start"], s["prefix"], c["prefix"], c["size"], O=s["O"])


OWN = dict(rotary=_own_rotary, fork=_own_fork, compact=_own_compact, shared=_own_shared)


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2501_16376_b200 import binding as sp
        return OWN[op](sp, state)
    return PLAIN[op](state)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    if case["op"] == "rotary":
        n = case["seqs"] * case["tokens"] * (case["heads"] + case["kv_heads"]) * case["head"]
        return dict(bytes=4 * n + 2 * case["rotary"], flops=(8 if case["norm"] else 4) * n)
    H, D, T = case["kv_heads"], case["head"], case["block"]
    block = H * (2 * T * D + 8)
    if case["op"] == "fork":
        B, L = case["groups"] * case["size"], case["length"]
        cols = (L + case["new"] + T - 1) // T
        copies = case["groups"] * (case["size"] - 1) if L % T else 0
        blocks = case["groups"] * ((L + T - 1) // T) + B * (cols - L // T) + 5
        return dict(bytes=2 * copies * block + 4 * blocks + 8 * B * cols, flops=0)
    if case["op"] == "compact":
        live = max(1, int(case["blocks"] * case["live"]))
        moved = live * (case["blocks"] - live) // case["blocks"]           # of a random pool, on average
        return dict(bytes=2 * moved * block + 8 * case["blocks"] + 8 * live, flops=0)
    rows, q = case["size"] * case["queries"] * case["group"], case["queries"] * case["group"]
    shared, lens = _shared_tokens(case), _lengths(case)
    tails = sum(n - shared[b // case["size"]] for b, n in enumerate(lens))
    io = 2 * 2 * case["groups"] * rows * H * D
    return dict(bytes=2 * D * H * (sum(shared) + tails) + io, flops=4 * D * H * (rows * sum(shared) + q * tails))


# ------------------------------------------------------------------ 64-bit values

def _exact_rotary(x, w, case, start, freq):
    y = x.double()
    D, r = y.shape[-1], case["rotary"]
    if w is not None:
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / D + 1e-6) * w.double()
    # a rotation is a product of complex numbers
    place = (start.double()[:, None] + torch.arange(y.shape[1], device=DEV, dtype=torch.float64))[:, :, None, None]
    unit = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), place * freq.double())
    out = y.clone()
    re, im = (slice(0, r, 2), slice(1, r, 2)) if case["pairs"] else (slice(0, r // 2), slice(r // 2, r))
    z = torch.complex(y[..., re].contiguous(), y[..., im].contiguous()) * unit
    out[..., re], out[..., im] = z.real, z.imag
    return out


def exact(case, seed):
    if case["op"] in ("fork", "compact"):                                  # whole numbers and copies
        return None
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return tuple(_exact_rotary(s[x], s[w], case, s["start"], s["freq"]) for x, w in (("Q", "wq"), ("K", "wk")))
    H, D, G, T, q = case["kv_heads"], case["head"], case["group"], case["block"], case["queries"]
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEV)
    table = s["table"].long()
    for b, length in enumerate(_lengths(case)):
        ids = table[b, :(length + T - 1) // T]
        K, V = (s[w][ids].view(torch.float8_e4m3fn).double() * s[w + "s"][ids].double()[..., None, None] for w in ("k", "v"))
        K, V = (x.transpose(0, 1).reshape(H, -1, D) for x in (K, V))
        for i in range(q):
            end = length - q + i + 1
            if end > 0:
                p = torch.softmax(s["Q"][b, i].double().view(H, G, D) @ K[:, :end].transpose(1, 2) / math.sqrt(D), -1)
                out[b, i] = (p @ V[:, :end]).view(H * G, D)
    return out
