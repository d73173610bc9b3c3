"""Plain 64-bit forms of the operators on the pool, and how far a kernel may be
from them, for the GPU tests.  Nothing here calls the library."""
from __future__ import annotations

import math

import numpy as np
import torch

F16, BF16, FP8, INT4 = 1, 2, 3, 4
NAMES = {F16: "f16", BF16: "bf16", FP8: "fp8", INT4: "int4"}
TORCH = {F16: torch.float16, BF16: torch.bfloat16, FP8: torch.float8_e4m3fn}
F64 = torch.float64


def half_step(t: torch.dtype) -> float:
    """What a rounding to t is off by at most, relative to the value."""
    return torch.finfo(t).eps / 2


def chunk_bytes(H, T, D, dtype):
    return 2 * H * T * D * {F16: 16, BF16: 16, FP8: 8, INT4: 5}[dtype] // 8


def codes_and_pairs(pool, shape):
    """Views of a 4-bit pool: words [L, N, 2, H, T, D/8] int32, (scale, base)
    [L, N, 2, H, T, D/32, 2] float16."""
    L, N, H, T, D, _ = shape
    rows = 2 * H * T
    c = pool[:L * N * rows * D * 5 // 8].view(L, N, rows * D * 5 // 8)
    words = c[:, :, :rows * D // 2].view(torch.int32).unflatten(2, (2, H, T, D // 8))
    pairs = c[:, :, rows * D // 2:].view(torch.float16).unflatten(2, (2, H, T, D // 32, 2))
    return words, pairs


def codes(words):
    """[..., D/8] int32 -> [..., D] codes, by the format's order in a word."""
    w = words.to(torch.int64)
    return torch.stack([(w >> ((e % 2) * 16 + (e // 2) * 4)) & 15 for e in range(8)], -1).flatten(-2)


def values(pool, shape):
    """What the pool stands for, float64 [L, N, 2, H, T, D]."""
    L, N, H, T, D, dtype = shape
    if dtype != INT4:
        n = L * N * chunk_bytes(H, T, D, dtype)
        return pool[:n].view(TORCH[dtype]).to(F64).view(L, N, 2, H, T, D)
    words, pairs = codes_and_pairs(pool, shape)
    p = pairs.to(F64)[..., None, :]
    c = codes(words).unflatten(-1, (D // 32, 32)).to(F64)
    return (p[..., 1] + (16 + c) * p[..., 0]).half().to(F64).flatten(-2)


def random_pool(shape, seed, extra=0, spread=1.0):
    """About normal values in every slot."""
    L, N, H, T, D, dtype = shape
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = L * N * chunk_bytes(H, T, D, dtype)
    pool = torch.zeros(n + extra, dtype=torch.uint8, device="cuda")
    if dtype == INT4:
        words, pairs = codes_and_pairs(pool, shape)
        words.copy_(torch.randint(-2 ** 31, 2 ** 31, words.shape, device="cuda", generator=gen)
                    .to(torch.int32))
        scale = torch.rand(pairs.shape[:-1], device="cuda", generator=gen) * 0.1 + 0.2
        pairs[..., 0] = scale * spread
        pairs[..., 1] = (torch.randn(scale.shape, device="cuda", generator=gen) * 0.3 - 2 -
                         16 * scale) * spread
    else:
        x = torch.randn(n // (1 if dtype == FP8 else 2), device="cuda", generator=gen) * spread
        pool[:n] = x.to(TORCH[dtype]).view(torch.uint8)
    return pool


def tables_for(ctx, T, N, seed, spare=0):
    """Disjoint random tables; `spare` more entries than a context needs."""
    rng = np.random.default_rng(seed)
    free = rng.permutation(N).astype(np.int32)
    out, at = [], 0
    for c in ctx:
        n = -(-c // T) + spare
        out.append(free[at:at + n])
        at += n
    assert at <= N
    return out


def poison_unused(pool, shape, tables, ctx, byte=0xFF):
    """Every slot that no context holds becomes NaN (all bits set)."""
    L, N, H, T, D, dtype = shape
    used = torch.zeros(N, T, dtype=torch.bool)
    for t, c in zip(tables, ctx):
        for i in range(-(-c // T)):
            used[int(t[i]), :min(T, c - i * T)] = True
    used = used.cuda()
    n = L * N * chunk_bytes(H, T, D, dtype)
    if dtype == INT4:
        words, pairs = codes_and_pairs(pool, shape)
        m = (~used)[None, :, None, None, :, None]
        words.masked_fill_(m, -1)
        pairs.view(torch.int16).masked_fill_(m[..., None], -1)
        return
    e = 1 if dtype == FP8 else 2
    rows = pool[:n].view(L, N, 2, H, T, D * e)
    rows.masked_fill_((~used)[None, :, None, None, :, None], byte)


def cached(vals, layer, table, ctx):
    """(keys, values) [H, ctx, D] of one sequence."""
    ids = torch.from_numpy(np.asarray(table)).long().cuda()[: max(1, len(table))]
    kv = vals[layer, ids].permute(1, 2, 0, 3, 4)
    return tuple(x.flatten(1, 2)[:, :ctx] for x in kv)


def attend(vals, layer, tables, ctx, new, q, k_scale=1.0, v_scale=1.0, scale=None):
    """(out, lse, sum of weights times |v|, sum of |q||k| at most), all float64, for
    packed queries [tokens, Hq, D]."""
    D = q.shape[2]
    scale = D ** -0.5 if scale is None else scale
    n, Hq = int(sum(new)), q.shape[1]
    out = torch.zeros(n, Hq, D, dtype=F64, device="cuda")
    mass, lse, reach = torch.zeros_like(out), out[..., 0].clone(), out[..., 0].clone()
    at = 0
    for t, c, m in zip(tables, ctx, new):
        if m == 0:
            continue
        k, v = cached(vals, layer, t, c)
        G = Hq // k.shape[0]
        x = q[at:at + m].to(F64)
        pos = torch.arange(c - m, c, device="cuda").repeat_interleave(G)
        hidden = torch.arange(c, device="cuda")[None] > pos[:, None]
        for h in range(k.shape[0]):
            sl = slice(h * G, (h + 1) * G)
            y = x[:, sl].reshape(m * G, D)
            s = (y @ k[h].T * (scale * k_scale)).masked_fill(hidden, -math.inf)
            l = torch.logsumexp(s, 1)
            w = (s - l[:, None]).exp()
            out[at:at + m, sl] = (w @ v[h] * v_scale).view(m, G, D)
            mass[at:at + m, sl] = (w @ v[h].abs() * v_scale).view(m, G, D)
            lse[at:at + m, sl] = l.view(m, G)
            far = (y.abs() @ k[h].abs().T).masked_fill(hidden, 0.0)
            reach[at:at + m, sl] = (far.amax(1) * abs(scale) * k_scale).view(m, G)
        at += m
    return out, lse, mass, reach


def attend_bounds(out, lse, mass, reach, D, longest, q_dtype, pool_dtype, vmax):
    """How far a kernel's (out, lse) may be off, element by element.  Scores: D products
    summed in fp32 (a step of 2^-23 each, the matrix instructions need not round to
    nearest), scaled and shifted: (D + 4) 2^-23 of the largest sum of |q||k| and the
    shift's rounding; where bf16 queries are taken to fp16, their smallest bits
    (2^-34 of the largest value).  A weight is off by that, by 2^-21 for exp2, and by half a step
    of the products' type; weights below fp16's normal range by 2^-25 / 2^6 / 2^-8
    of the largest.  Sums of n terms: (n + 16) 2^-24 (split over at least 16 lanes'
    partial sums where n is large).  The result's own rounding."""
    m = torch.float16 if pool_dtype == INT4 else q_dtype
    ds = (D + 6) * 2.0 ** -23 * reach + lse.abs() * 2.0 ** -22 + 2.0 ** -21
    sums = (longest / 16 + 64) * 2.0 ** -23
    weight = ds * 1.01 + half_step(m) + sums
    o = mass * (weight + ds + sums)[..., None] * 1.02 + out.abs() * half_step(q_dtype) + \
        longest * 2.0 ** -23 * vmax * 2.0 ** -6 + 2.0 ** -25
    return o, ds * 1.02 + 2 * sums + lse.abs() * 2.0 ** -22


def rotate(x, pos, rope, interleaved):
    """(float64 rotated [tokens, heads, D], what the two products of each value sum to in
    size): the first rope.shape[1] values of a head are turned."""
    R = rope.shape[1]
    row = rope[pos.long()].to(F64)
    co, si = row[:, None, :R // 2], row[:, None, R // 2:]
    y, size = x.to(F64).clone(), x.to(F64).abs()
    a, b = ((slice(0, R, 2), slice(1, R, 2)) if interleaved
            else (slice(0, R // 2), slice(R // 2, R)))
    u, w = x[..., a].to(F64), x[..., b].to(F64)
    y[..., a], y[..., b] = u * co - w * si, w * co + u * si
    size[..., a] = (u * co).abs() + (w * si).abs()
    size[..., b] = (w * co).abs() + (u * si).abs()
    return y, size


def rope_table(rows, R, base=10000.0):
    angle = torch.arange(rows, dtype=F64)[:, None] * base ** (-torch.arange(0, R, 2, dtype=F64) / R)
    return torch.cat([angle.cos(), angle.sin()], 1).float().cuda()


def positions(ctx, new):
    return np.concatenate([np.arange(c - n, c) for c, n in zip(ctx, new)] or [[]]).astype(np.int64)


def slots(tables, ctx, new, T):
    p = positions(ctx, new)
    ids = [np.asarray(t)[np.arange(c - n, c) // T] for t, c, n in zip(tables, ctx, new)]
    return (torch.from_numpy(np.concatenate(ids or [[]]).astype(np.int64)).cuda(),
            torch.from_numpy(p % T).cuda())


def assert_within(got, want, bound, what):
    d = (got.to(F64) - want).abs()
    bad = ~(d <= bound)
    if bool(bad.any()):
        i = int(bad.flatten().nonzero()[0])
        raise AssertionError(
            f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: "
            f"{float(got.flatten()[i])} != {float(want.flatten()[i])} "
            f"(bound {float(torch.broadcast_to(bound, d.shape).flatten()[i]):.3g})")
