"""What the operators on the paged KV pool are measured on: one pass of each
call that a serving engine issues for a layer, through the package's public
entry points.

  append   a batch's new keys and values written into the pool, the keys and
           the queries rotated by their positions on the way
  attend   causal attention of the batch's new tokens over the pool
  layer    the two in turn, as a layer of a model issues them

A case names a pool (layers, KV heads, tokens per block, head size, element
type), the query heads and their type, and the batch: ``prompts`` sequences
with contexts spread evenly in ratio between ``min_tokens`` and ``max_tokens``,
each with ``new`` tokens of its own in the call (0: all of them, a prompt that
is computed whole), and, where ``chunk`` is not 0, one more sequence that
computes ``chunk`` tokens at the end of a context of ``chunk_context``.  Block
tables are a random permutation of the pool, as a free list that has been in
use for a while leaves them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

F32, F64 = torch.float32, torch.float64
TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
BITS = {"f16": 16, "bf16": 16, "fp8": 8, "int4": 5}   # int4: 4, and 32 for each 32 values
GROUP = 32                                            # values with one scale and base (int4)
LARGEST4 = 16384.0                                    # what a 4-bit pool holds at most
LARGEST8 = 448.0                                      # what an e4m3 pool holds at most


def _case(name, op, pool, dtype, q_heads, q_dtype, prompts, min_tokens, max_tokens, new,
          chunk=0, chunk_context=0, interleaved=False):
    heads, block_tokens, head_dim = pool
    return {"name": name, "op": op, "layers": 2, "heads": heads, "block_tokens": block_tokens,
            "head_dim": head_dim, "dtype": dtype, "q_heads": q_heads, "q_dtype": q_dtype,
            "prompts": prompts, "min_tokens": min_tokens, "max_tokens": max_tokens, "new": new,
            "chunk": chunk, "chunk_context": chunk_context, "interleaved": interleaved}


def listed():
    p8, p70, tp8 = (8, 16, 128), (8, 16, 128), (1, 16, 128)
    return [
        # One chat of an 8B model writes the key and value of its next token:
        # the smallest append, all latency.
        _case("append_one", "append", p8, "bf16", 32, "bf16", 1, 512, 512, 1),
        # A full decode batch of an 8B model on an fp8 pool.
        _case("append_batch_fp8", "append", p8, "fp8", 32, "bf16", 256, 64, 8192, 1),
        # A long prompt of a 70B model is computed whole.
        _case("append_prompt", "append", p70, "bf16", 64, "bf16", 1, 16384, 16384, 0),
        # Prompts of ragged lengths written into a 4-bit pool.
        _case("append_ragged_int4", "append", p8, "int4", 32, "f16", 13, 17, 3001, 0,
              interleaved=True),
        # One short chat answers: the smallest attention.
        _case("attend_one", "attend", p8, "f16", 32, "f16", 1, 512, 512, 1),
        # The decode step of a batch of chats of very different lengths.
        _case("attend_chats", "attend", p8, "bf16", 32, "bf16", 64, 128, 8192, 1),
        # One 32768-token prompt of a 70B model decodes: few rows, a long axis.
        _case("attend_long", "attend", p70, "bf16", 64, "bf16", 1, 32768, 32768, 1),
        # Decode batches of the same shape in 8 and in 4 bits.
        _case("attend_fp8", "attend", p8, "fp8", 32, "bf16", 64, 128, 8192, 1),
        _case("attend_int4", "attend", p8, "int4", 32, "bf16", 64, 128, 8192, 1),
        # One rank of a 70B model over a node, a long document in 4 bits.
        _case("attend_long_int4", "attend", tp8, "int4", 8, "f16", 3, 30001, 131072, 1),
        # A prompt of an 8B model computed whole: matrix products all through.
        _case("attend_prompt", "attend", p8, "bf16", 32, "bf16", 1, 8192, 8192, 0),
        # A chunked prefill beside a decode batch on a 4-bit pool.
        _case("layer_chunk_int4", "layer", p8, "int4", 32, "bf16", 40, 100, 4000, 1,
              chunk=1021, chunk_context=9000),
    ]


LARGEST = 1.2e12        # operations of a case
LARGEST_BYTES = 2 << 30
LARGEST_PLAIN = 3 << 28  # scores, or keys, that the plain form holds at once


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(("append", "attend", "attend", "attend", "layer"))
        dtype = rng.choice(("f16", "bf16", "bf16", "fp8", "int4", "int4"))
        q_dtype = dtype if dtype in ("f16", "bf16") else rng.choice(("f16", "bf16"))
        heads, q_heads, head_dim = rng.choice(
            ((8, 32, 128), (8, 64, 128), (1, 8, 128), (2, 16, 128), (4, 28, 128), (5, 40, 128),
             (32, 32, 128), (8, 64, 64), (3, 15, 64), (12, 12, 64), (1, 71, 64), (4, 8, 256)))
        pool = (heads, rng.choice((8, 16, 16, 32)), head_dim)
        kind = rng.choice(("decode", "decode", "few", "whole", "chunk"))
        prompts = _log_int(rng, 1, 256)
        most = _log_int(rng, 1, 131072 if kind in ("decode", "few") else 8192)
        least = max(1, int(most / rng.uniform(1.0, 64.0)))
        new = {"decode": 1, "few": rng.randint(2, 6), "whole": 0, "chunk": 1}[kind]
        chunk = _log_int(rng, 16, 4096) if kind == "chunk" else 0
        c = _case("", op, pool, dtype, q_heads, q_dtype, prompts, max(least, new), max(most, new),
                  new, chunk, chunk + _log_int(rng, 1, 16384) if chunk else 0,
                  rng.random() < 0.3)
        del c["name"]
        w = work(c)
        ctx, news = _lengths(c)
        plain = max(len(g) * max(ctx[g]) * max(q_heads * max(news[g]), 2 * heads * head_dim)
                    for g in _groups(c))
        pool_bytes = c["layers"] * sum(-(-ctx // pool[1])) * pool[1] * heads * head_dim * BITS[dtype] // 4
        if op == "append" and dtype == "int4" and pool_bytes > (64 << 20):
            continue   # all of a 4-bit pool is turned into the values it stands for
        if w["flops"] <= LARGEST and w["bytes"] <= LARGEST_BYTES and plain <= LARGEST_PLAIN and \
                pool_bytes <= (8 << 30) and sum(news) <= 65536:
            return c


# -- inputs -------------------------------------------------------------------

def _lengths(case):
    """(contexts, new tokens) of the sequences, int64 arrays."""
    n, lo, hi = case["prompts"], case["min_tokens"], case["max_tokens"]
    ctx = [int(round(lo * (hi / lo) ** (i / max(1, n - 1)))) for i in range(n)]
    new = [case["new"] or c for c in ctx]
    if case["chunk"]:
        ctx.append(case["chunk_context"])
        new.append(case["chunk"])
    return np.asarray(ctx), np.asarray(new)


def _groups(case):
    """The sequences that the plain form pads to one length."""
    n = case["prompts"]
    return [np.arange(n)] + ([np.array([n])] if case["chunk"] else [])


def _values(nbytes, dtype, gen):
    """KV values as a model leaves them: about normal."""
    if dtype in ("f16", "bf16"):
        return torch.empty(nbytes // 2, dtype=TORCH[dtype], device="cuda").normal_(generator=gen) \
            .view(torch.uint8)
    out = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    step = 1 << 28
    for at in range(0, nbytes, step):
        part = out[at:at + step]
        part.copy_(torch.empty(part.numel(), dtype=torch.float16, device="cuda")
                   .normal_(generator=gen).to(torch.float8_e4m3fn).view(torch.uint8))
    return out


def _codes4(pool, case):
    """The two parts of a 4-bit pool: code bytes [L, N, 2, H, T, D/2], and
    (scale, base) pairs [L, N, 2, H, T, D/32, 2]."""
    H, T, D = case["heads"], case["block_tokens"], case["head_dim"]
    rows = 2 * H * T
    chunks = pool.view(case["layers"], -1, rows * D * 5 // 8)
    codes = chunks[:, :, :rows * D // 2].unflatten(2, (2, H, T, D // 2))
    pairs = chunks[:, :, rows * D // 2:].view(torch.float16).unflatten(2, (2, H, T, D // GROUP, 2))
    return codes, pairs


def _fill4(case, nbytes, gen):
    """A 4-bit pool of about normal values: random codes, and the scales and
    bases that normal groups have."""
    pool = torch.randint(0, 1 << 31, (nbytes // 4,), dtype=torch.int32, device="cuda",
                         generator=gen)
    pool = (pool ^ (pool << 7)).view(torch.uint8)
    pairs = _codes4(pool, case)[1]
    scale = torch.empty(pairs.shape[:-1], device="cuda").normal_(0.28, 0.03, generator=gen)
    pairs[..., 0] = scale
    pairs[..., 1] = torch.empty_like(scale).normal_(-2.1, 0.3, generator=gen) - 16 * scale
    return pool


class _State:
    """Inputs and what a program keeps; closes the pool, and the batch with it, when it is
    dropped."""

    def __del__(self):
        kv = getattr(self, "kv", None)
        if kv is not None:
            kv.close()


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    x = _State()
    x.case = case
    L, H, T, D = case["layers"], case["heads"], case["block_tokens"], case["head_dim"]
    Hq, dt = case["q_heads"], TORCH[case["q_dtype"]]
    x.ctx, x.new = _lengths(case)
    counts = -(-x.ctx // T)
    N = int(sum(counts)) + 3
    free = rng.permutation(N).astype(np.int32)
    ends = np.cumsum(counts)
    x.tables = [free[e - n:e] for e, n in zip(ends, counts)]
    nbytes = L * N * 2 * H * T * D * BITS[case["dtype"]] // 8
    x.pool = _fill4(case, nbytes, gen) if case["dtype"] == "int4" else \
        _values(nbytes, case["dtype"], gen)
    x.layer = 1
    x.k_scale, x.v_scale = (0.75, 1.25) if case["dtype"] == "fp8" else (1.0, 1.0)
    tokens = int(sum(x.new))
    x.tokens = tokens
    # What a fused projection leaves: queries, keys and values side by side.
    qkv = torch.empty(tokens, Hq + 2 * H, D, dtype=dt, device="cuda").normal_(generator=gen)
    x.q, x.k, x.v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    most = int(max(x.ctx))
    angle = torch.arange(most, dtype=F64, device="cuda")[:, None] * \
        10000.0 ** (-torch.arange(0, D, 2, dtype=F64, device="cuda") / D)
    x.rope = torch.cat([angle.cos(), angle.sin()], 1).float()
    # Where each new token goes, and each sequence's blocks, padded.
    x.pos = torch.from_numpy(np.concatenate([np.arange(c - n, c) for c, n in zip(x.ctx, x.new)])) \
        .cuda()
    x.block = torch.from_numpy(np.concatenate(
        [t[np.arange(c - n, c) // T] for t, c, n in zip(x.tables, x.ctx, x.new)])).long().cuda()
    x.slot = x.pos % T
    first = np.cumsum(x.new) - x.new
    x.groups = []
    for g in _groups(case):
        padded = np.zeros((len(g), max(counts[g])), dtype=np.int64)
        for i, s in enumerate(g):
            padded[i, :counts[s]] = x.tables[s]
        at = first[g][:, None] + np.arange(max(x.new[g]))
        there = np.arange(max(x.new[g])) < x.new[g][:, None]
        pos = (x.ctx - x.new)[g][:, None] + np.arange(max(x.new[g]))
        x.groups.append(tuple(torch.from_numpy(a).cuda() for a in
                              (padded, np.where(there, at, first[g][:, None]), there, pos)))
    return x


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2407_21255_amd import aqua
        L, H, T, D = case["layers"], case["heads"], case["block_tokens"], case["head_dim"]
        kinds = {"f16": aqua.AQUA_F16, "bf16": aqua.AQUA_BF16, "fp8": aqua.AQUA_FP8_E4M3,
                 "int4": aqua.AQUA_INT4}
        blocks = sum(len(t) for t in s.tables)
        s.kv = aqua.KVPool((L, blocks + 3, H, T, D, kinds[case["dtype"]]), s.pool)
        s.batch = aqua.KVBatch(s.kv, case["q_heads"], max_seqs=len(s.tables),
                               max_tokens=s.tokens, max_blocks=blocks)
        s.batch.set(s.tables, s.ctx, s.new)
    torch.cuda.synchronize()
    return s


# -- one pass -----------------------------------------------------------------

def run(s):
    op = s.case["op"]
    if op == "append":
        q = _append(s)
        return {"q": q, "pool": _held(s)}
    if op == "attend":
        return _attend(s, s.q)
    return _attend(s, _append(s))


def _held(s):
    """What the pool stands for after an append."""
    if s.case["dtype"] == "int4":
        return _decode4(*_codes4(s.pool, s.case))
    return s.pool.view(TORCH[s.case["dtype"]])


def _append(s):
    if own:
        return s.batch.append(s.layer, s.k, s.v, q=s.q, rope=s.rope,
                              interleaved=s.case["interleaved"], k_scale=s.k_scale,
                              v_scale=s.v_scale)
    turn = s.rope[s.pos][:, None]
    q, k = (_rotate(t.float(), turn, s.case["interleaved"]) for t in (s.q, s.k))
    _store(s, 0, k, s.k_scale)
    _store(s, 1, s.v.float(), s.v_scale)
    return q.to(s.q.dtype)


def _rotate(t, turn, interleaved):
    cos, sin = turn.chunk(2, -1)
    if interleaved:
        a, b = t[..., 0::2], t[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    a, b = t.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _store(s, which, t, scale):
    c = s.case
    L, H, T, D = c["layers"], c["heads"], c["block_tokens"], c["head_dim"]
    if c["dtype"] == "int4":
        codes, pairs = _codes4(s.pool, c)
        w, p = _encode4(t)
        codes[s.layer, s.block, which, :, s.slot] = w
        pairs[s.layer, s.block, which, :, s.slot] = p
        return
    if c["dtype"] == "fp8":
        t = (t / scale).clamp(-LARGEST8, LARGEST8)
    rows = t.to(TORCH[c["dtype"]]).view(torch.uint8)
    pool = s.pool.view(L, -1, 2, H, T, rows.shape[-1])
    pool[s.layer, s.block, which, :, s.slot] = rows


# A 4-bit pool holds a group of 32 values as codes of 0 to 15 with a scale and
# a base in 16 bits; a code stands for base + (16 + code) * scale.  Of each 8
# values, the even ones are in the low 16 bits of a word and the odd ones in
# the high 16 bits.
SHIFTS = (0, 16, 4, 20, 8, 24, 12, 28)


def _encode4(t):
    g = t.clamp(-LARGEST4, LARGEST4).unflatten(-1, (-1, GROUP))
    low = g.amin(-1, keepdim=True)
    scale = ((g.amax(-1, keepdim=True) - low) / 15).half()
    base = (low - scale.float() * 16).half()
    step = torch.where(scale > 0, scale.float(), torch.ones_like(low))
    code = (((g - base.float()) / step).round() - 16).clamp(0, 15).int()
    shift = torch.tensor(SHIFTS, dtype=torch.int32, device=t.device)
    words = (code.unflatten(-1, (-1, 8)) << shift).sum(-1, dtype=torch.int32)
    return words.flatten(-2).contiguous().view(torch.uint8), torch.cat([scale, base], -1)


def _decode4(codes, pairs):
    """The values, float16, in the shape [..., D]."""
    low, high = codes & 15, codes >> 4
    # Byte b of a word holds value 2b' + (b >= 2) of each 4-bit half.
    both = torch.stack([low, high], -1).unflatten(-2, (-1, 2, 2))      # [.., 8s, odd, byte, nibble]
    code = both.movedim(-3, -1).flatten(-4).unflatten(-1, (-1, GROUP))
    scale, base = pairs[..., :1].float(), pairs[..., 1:].float()
    return (base + (16 + code) * scale).half().flatten(-2)


def _cached(s, which, blocks):
    """Keys or values of a table's blocks, [sequences, heads, tokens, D]."""
    c = s.case
    L, H, T, D = c["layers"], c["heads"], c["block_tokens"], c["head_dim"]
    if c["dtype"] == "int4":
        codes, pairs = _codes4(s.pool, c)
        t = _decode4(codes[s.layer, blocks, which], pairs[s.layer, blocks, which]).float()
    else:
        t = s.pool.view(TORCH[c["dtype"]]).view(L, -1, 2, H, T, D)[s.layer, :, which]
        t = t.view(torch.uint8)[blocks].view(TORCH[c["dtype"]]).float()
    return t.movedim(2, 1).flatten(2, 3)


def _attend(s, q):
    if own:
        out, lse = s.batch.attend(s.layer, q, lse=True, k_scale=s.k_scale, v_scale=s.v_scale)
        return {"out": out, "lse": lse}
    c = s.case
    H, D = c["heads"], c["head_dim"]
    G = c["q_heads"] // H
    outs, sums = [], []
    for blocks, rows, there, pos in s.groups:
        k, v = _cached(s, 0, blocks), _cached(s, 1, blocks)
        n, m = there.shape
        x = q[rows].float().view(n, m, H, G, D).permute(0, 2, 3, 1, 4).reshape(n, H, G * m, D)
        far = torch.arange(k.shape[2], device=q.device) > pos[:, :, None]       # [n, m, tokens]
        y = (x @ k.transpose(-1, -2)).mul_(s.k_scale / math.sqrt(D)).unflatten(2, (G, m))
        y.masked_fill_(far[:, None, None], -math.inf)
        top = y.amax(-1, keepdim=True)
        y.sub_(top).exp_()
        total = y.sum(-1, keepdim=True)
        o = (y.flatten(2, 3) @ v).unflatten(2, (G, m)) * (s.v_scale / total)
        outs.append(o.permute(0, 3, 1, 2, 4).flatten(2, 3)[there])
        sums.append((top + total.log()).squeeze(-1).permute(0, 3, 1, 2).flatten(2, 3)[there])
    return {"out": torch.cat(outs).to(q.dtype), "lse": torch.cat(sums)}


# -- what a pass cannot do without ---------------------------------------------

def work(case):
    ctx, new = _lengths(case)
    tokens, D, H, Hq = int(sum(new)), case["head_dim"], case["heads"], case["q_heads"]
    row = 2 * H * D * BITS[case["dtype"]] / 8      # a token's key and value in the pool
    bytes_, flops = 0.0, 0.0
    if case["op"] in ("append", "layer"):
        places = int(max(new)) if case["new"] == 0 else min(tokens, int(max(ctx)))
        bytes_ += tokens * (2 * (2 * Hq + 2 * H) * D + row) + places * 4 * D
        flops += tokens * 3.0 * (Hq + H) * D
    if case["op"] in ("attend", "layer"):
        pairs = sum(int(n) * (int(c) - int(n)) + int(n) * (int(n) + 1) // 2
                    for c, n in zip(ctx, new))
        bytes_ += float(sum(int(c) for c in ctx)) * row + tokens * Hq * (4 * D + 4)
        flops += 4.0 * pairs * Hq * D
    return {"bytes": bytes_, "flops": flops}


# -- the same in 64 bits --------------------------------------------------------

def exact(case, seed):
    """From the definitions, sequence by sequence and head by head."""
    x = _inputs(case, seed)
    L, H, T, D = case["layers"], case["heads"], case["block_tokens"], case["head_dim"]
    Hq = case["q_heads"]
    turned = {}
    if case["op"] in ("append", "layer"):
        c, s = x.rope[x.pos].to(F64).split(D // 2, 1)
        for name in ("q", "k"):
            t = getattr(x, name).to(F64)
            first = torch.arange(0, D, 2) if case["interleaved"] else torch.arange(D // 2)
            second = first + (1 if case["interleaved"] else D // 2)
            r = torch.empty_like(t)
            r[:, :, first] = t[:, :, first] * c[:, None] - t[:, :, second] * s[:, None]
            r[:, :, second] = t[:, :, first] * s[:, None] + t[:, :, second] * c[:, None]
            turned[name] = r
        fresh = [_as_held(turned["k"], case, x.k_scale), _as_held(x.v.to(F64), case, x.v_scale)]
    if case["op"] == "append":
        pool = _pool64(x, case)
        for which in (0, 1):
            pool[x.layer, x.block, which, :, x.slot] = fresh[which]
        pool = pool if case["dtype"] == "int4" else pool.flatten()
        return {"q": turned["q"], "pool": pool}
    q = turned["q"].to(x.q.dtype).to(F64) if turned else x.q.to(F64)
    out = torch.empty(x.tokens, Hq, D, dtype=F64, device="cuda")
    lse = torch.empty(x.tokens, Hq, dtype=F64, device="cuda")
    at = 0
    for table, n_ctx, n_new in zip(x.tables, x.ctx, x.new):
        ids = torch.from_numpy(table).long().cuda()
        kv = _pool64(x, case, ids)[0]                      # [blocks, 2, H, T, D]
        kv = kv.permute(1, 2, 0, 3, 4).reshape(2, H, -1, D)[:, :, :n_ctx]
        if turned:
            for which in (0, 1):
                held = fresh[which][at:at + n_new]
                if case["dtype"] not in ("int4",):
                    held = held.to(TORCH[case["dtype"]]).to(F64)
                kv[which, :, n_ctx - n_new:] = held.transpose(0, 1)
        kv[0] *= x.k_scale
        kv[1] *= x.v_scale
        for lo in range(0, n_new, 1024):
            hi = min(n_new, lo + 1024)
            seen = torch.arange(n_ctx, device="cuda")[None] <= \
                (n_ctx - n_new + torch.arange(lo, hi, device="cuda"))[:, None]
            for h in range(Hq):
                g = h * H // Hq
                z = q[at + lo:at + hi, h] @ kv[0, g].T / D ** 0.5
                z = z.masked_fill(~seen, -math.inf)
                sums = torch.logsumexp(z, 1)
                lse[at + lo:at + hi, h] = sums
                out[at + lo:at + hi, h] = (z - sums[:, None]).exp() @ kv[1, g]
        at += n_new
    return {"out": out, "lse": lse}


def _as_held(t, case, scale):
    """Rows as the pool holds them, before the rounding to its type (int4: after it)."""
    if case["dtype"] == "fp8":
        return (t / scale).clamp(-LARGEST8, LARGEST8)
    if case["dtype"] != "int4":
        return t
    g = t.reshape(*t.shape[:-1], -1, GROUP).clamp(-LARGEST4, LARGEST4)
    lo, hi = g.min(-1).values, g.max(-1).values
    scale = ((hi - lo) / 15).half().to(F64)
    base = (lo - 16 * scale).half().to(F64)
    step = torch.where(scale > 0, scale, torch.ones_like(scale))[..., None]
    code = (torch.round((g - base[..., None]) / step) - 16).clamp(0, 15)
    return (base[..., None] + (16 + code) * scale[..., None]).half().to(F64).reshape(t.shape)


def _pool64(x, case, ids=None):
    """The pool's values [layers, blocks, 2, H, T, D] (with ``ids``: of those
    blocks of the layer) in 64 bits."""
    L, H, T, D = case["layers"], case["heads"], case["block_tokens"], case["head_dim"]
    chunks = x.pool.view(L, -1, 2 * H * T * D * BITS[case["dtype"]] // 8)
    if ids is not None:
        chunks = chunks[x.layer:x.layer + 1, ids]
    if case["dtype"] != "int4":
        return chunks.view(TORCH[case["dtype"]]).to(F64).unflatten(2, (2, H, T, D))
    rows = 2 * H * T
    words = chunks[:, :, :rows * D // 2].contiguous().view(torch.int32).to(torch.int64)
    code = torch.stack([(words >> s) & 15 for s in (0, 16, 4, 20, 8, 24, 12, 28)], -1)
    pair = chunks[:, :, rows * D // 2:].contiguous().view(torch.float16).to(F64)
    pair = pair.unflatten(2, (2, H, T, D // GROUP, 2))
    code = code.flatten(2).unflatten(2, (2, H, T, D // GROUP, GROUP))
    return (pair[..., 1:] + (16 + code) * pair[..., :1]).half().to(F64).flatten(-2)
